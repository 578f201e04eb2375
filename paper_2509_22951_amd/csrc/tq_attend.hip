// Attention of one new token per row over a paged cache (tq_attend).
//
// A wavefront takes 32 tokens of one key/value head at a time and up to 8 of the query heads that share it.  Both products run on
// v_mfma_f32_16x16x32_bf16, keys and values go from memory to registers in the shape the instruction wants, and nothing passes
// through LDS or between lanes but the softmax maxima:
//   logits^T [token][head] = K [token][dim] Q^T: lane l supplies token l % 16 and 8 neighbouring dims (16 bytes of a key).
//   out^T [dim][head] = V^T [dim][token] P^T: the lane that got the logits of tokens 4g..4g+3 of both 16-token blocks (g = l / 16)
//   supplies the same tokens as its 8 values of the contraction, so P is already where it is needed; it loads DIM / 16
//   neighbouring dims of those 8 tokens' values and transposes that square in its registers (one v_perm per pair).
// The 16 columns are 8 heads twice: column c holds the upper 8 bits of head c's mantissas, column c + 8 the next 8, and a second
// product has the last 8 beside zeros, so that q and p enter with all of fp32's 24 bits.  (p with 16 of them, one product: the same time within
// 2 %, 200 tokens 5.8 us in place of 6.0; but up to 2^-17 of each weight off, more than all else together: a result next to the
// middle of two bf16 values went to the other one in one of a thousand.)
#include <algorithm>

#include "tq_cache_view.h"
#include "tq_strip_decode.h"

namespace tq {
namespace {

constexpr int kAttendWaves = 8, kAttendThreads = kAttendWaves * 64, kTile = 32, kHeads = 8;   // kHeads: query heads of a workgroup
constexpr uint32_t kUnit = kAttendWaves * kTile;                          // tokens that a workgroup takes at a time
constexpr uint32_t kMaxGroups = 256, kCluster = 16;   // workgroups of a launch (one per compute unit); parts that are joined at a time
constexpr uint64_t kPassing = 8 << 20;   // bytes of keys and values
constexpr uint32_t kMostAligned = 16;   // units of a share (8 and 32: no difference seen)
constexpr uint32_t kCounters = 2 * (kMaxGroups / kCluster) + kMaxGroups;
constexpr float kLog2e = 1.4426950408889634f;

struct AttendView {
  const void* q;
  uint16_t* out;
  const int32_t *seqs, *lengths;
  // [cluster][2], then [workgroup]: the workgroups, or clusters, whose part of a (row, chunk) is in the partials; zero between calls.  Of a
  // (row, chunk) that is cut the workgroup in which it begins, which begins no other one that reaches beyond it: the same places for
  // all rows, heads and lengths, so that calls of any of them may follow each other on one workspace.
  uint32_t* arrived;
  float* partials;     // [workgroup][2]: kHeads x head_dim sums, then maximum and total of every head
  float* logits;       // [row][head][capacity], in units of log 2 (accumulate)
  float2* stats;       // [row][head]: maximum and 1 / total of the whole row (accumulate)
  uint64_t q_stride, out_stride;
  float scale;         // times log2(e)
  uint32_t rows, heads, group, chunks, q16, out_by4;   // chunks: of up to kHeads query heads that share a key/value head, of all of these
};

__device__ __forceinline__ uint32_t ror8(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x128, 0xf, 0xf, true); }   // v of the lane 8 columns on
__device__ __forceinline__ float ror8_sum(float v) { return v + __uint_as_float(ror8(__float_as_uint(v))); }

__device__ __forceinline__ uint32_t row_length(const CacheView& c, const AttendView& a, uint32_t r, uint32_t* seq) {
  const int32_t s = a.seqs ? a.seqs[r] : (int32_t)r;
  *seq = (uint32_t)s < c.n_seqs ? (uint32_t)s : 0;
  return (uint32_t)s < c.n_seqs ? (uint32_t)min(max(a.lengths[r], 0), (int32_t)c.capacity) : 0;
}

typedef __attribute__((address_space(1), aligned(2))) const uint32_t global_cu32_any;

template <int DIM, bool INT8>
struct Tile {
  static constexpr int kSteps = DIM / 32, kVals = DIM / 16;   // contraction steps of the logits; a lane's dims of a value
  static constexpr int kLoads = INT8 ? kSteps / 2 : kSteps;   // 16-byte loads of a key
  static constexpr int kValWords = INT8 ? kVals / 4 : kVals / 2;
  uint32_t k[2][4 * kLoads], v[8][kValWords];
  float4 ks[2], vs[2];
};

// Where loads that pass the caches by are faster: no byte is loaded twice.  Through the caches and past them, us: 16 x 16384 tokens of 128 dims
// 180 and 166, 16 x 32768 of 64 190 and 176, of 128 in 8 bits 201 and 188, 4 x 32768 of 256 99 and 93; 1 x 16000 of 96 16.2 and 15.5 (2 x 50000
// 37 and 38); but of 80 and 48, whose rows begin anywhere in a line, 16 x 8000 64 and 72, 42 and 43, and of 64 in 8 bits no gain.
template <int DIM, bool INT8>
constexpr bool kPasses = DIM >= 128 || !INT8;

template <int WORDS, bool PASSES>
__device__ __forceinline__ void load_words(uint32_t* to, const char* from) {
  constexpr int kWords = WORDS % 4 ? WORDS : 4;
  typedef uint32_t words __attribute__((ext_vector_type(kWords)));
#pragma unroll
  for (int w = 0; w < WORDS; w += kWords) {
    const words* at = (const words*)(from + 4 * w);
    words d;
    if constexpr (PASSES) d = __builtin_nontemporal_load(at);
    else d = *at;
#pragma unroll
    for (int i = 0; i < kWords; ++i) to[w + i] = kWords == 1 ? *(const uint32_t*)&d : d[i];
  }
}

__device__ __forceinline__ uint32_t units_of(uint32_t length) { return max((length + kUnit - 1) / kUnit, 1u); }   // (an empty row is written too)

// The largest of 64 lanes, in the last one.
__device__ __forceinline__ uint32_t max_of_lanes(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xf, 0xf, true));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xf, 0xf, true));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xf, 0xf, true));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xf, 0xf, true));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xa, 0xf, false));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xc, 0xf, false));
  return v;
}

struct Segment {   // the part of a (row, chunk) that lies in a workgroup's share
  uint32_t r, seq, kv, first_head, n_heads, pair_first, units, begin, end, rounds;   // rounds of kUnit tokens, the same for every wavefront
};

// A wavefront's tokens of a segment once more, a product per value as the formula has them, so that infinities give what they give there.
// The results replace those in LDS (and the logits).  32 tokens at a time, two lanes per key, then a lane per dim of the values: slow, and
// only for what is not finite (8 x 8192 tokens, 8 heads of 128: 47 us, with one infinite key 352, with infinities in all keys 1017).  What it
// needs is read again from the kernel's arguments, and nothing of it computed ahead: the tile loop has no registers for it.
template <int DIM, bool INT8, bool TRACK>
__device__ __forceinline__ void take_again(const Segment& s, uint32_t lane, uint32_t wave, float* lds_sum, float* lds_max, float* lds_total) {
  typedef __attribute__((address_space(4))) const char constant_char;
  typedef __attribute__((address_space(4))) const CacheView constant_cache;
  typedef __attribute__((address_space(4))) const AttendView constant_attend;
  static_assert(sizeof(CacheView) % alignof(AttendView) == 0, "the kernel's arguments lie side by side");
  constexpr uint32_t kOwn = (DIM + 63) / 64;
  constant_char* args = (constant_char*)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(args), "+v"(lane));
  constant_cache& c = *(constant_cache*)args;
  constant_attend& a = *(constant_attend*)(args + sizeof(CacheView));
  const uint32_t D = c.head_dim, slot_bytes = (INT8 ? 1 : 2) * (uint32_t)c.slot_stride, n_pages = c.n_pages, mask = (1u << c.page_shift) - 1, t = lane % 32;
  const bool q16 = a.q16;
  const float scale = a.scale;
  const char *keys = c.k, *values = c.v;
  const float *k_scale = c.k_scale, *v_scale = c.v_scale;
  const int32_t* table = c.tables + (uint64_t)s.seq * c.table_stride;
  __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0): the logits stored before
#pragma unroll 1
  for (uint32_t h = 0; h < s.n_heads; ++h) {
    const uint64_t q_at = s.r * a.q_stride + (s.first_head + h) * D;
    float m = -INFINITY, sum_p = 0.f, sum[kOwn] = {};
#pragma unroll 1
    for (uint32_t round = 0; round < s.rounds; ++round) {
      const uint32_t tile = s.begin + round * kUnit + wave * kTile, slot = tile + t;
      uint32_t page = n_pages;
      if (slot < s.end) page = (uint32_t)table[slot >> c.page_shift];
      const bool there = page < n_pages;
      const uint64_t at = (INT8 ? 1 : 2) * ((there ? page : 0) * c.page_stride + s.kv * c.head_stride) + (uint64_t)(slot & mask) * slot_bytes;
      const uint64_t mark = (((uint64_t)(there ? page : 0) * c.kv_heads + s.kv) << c.page_shift) + (slot & mask);
      const char* key = keys + at;
      float l = 0.f;
#pragma unroll 1
      for (uint32_t i = 0, d = lane < 32 ? 0 : D / 2; i < D / 2; ++i, ++d) {
        const float of_q = (q16 ? bf16_value(((const uint16_t*)a.q)[q_at + d]) : ((const float*)a.q)[q_at + d]) * scale;
        l = fmaf(of_q, INT8 ? (float)((const int8_t*)key)[d] : bf16_value(((const uint16_t*)key)[d]), l);
      }
      l += __shfl_xor(l, 32);
      if constexpr (INT8) l *= k_scale[mark];
      if (!there) l = -INFINITY;
      if (TRACK && lane < 32 && slot < s.end) a.logits[((uint64_t)s.r * a.heads + s.first_head + h) * c.capacity + slot] = l;
      const float top = fmaxf(m, group_max<32>(l)), base = top == -INFINITY ? 0.f : top, shrink = __builtin_amdgcn_exp2f(m - base);
      float p = __builtin_amdgcn_exp2f(l - base);
      m = top;
      sum_p = fmaf(sum_p, shrink, group_sum<32>(p));
      if constexpr (INT8) p = there ? p * v_scale[mark] : 0.f;
#pragma unroll
      for (uint32_t i = 0; i < kOwn; ++i) sum[i] *= shrink;
      const uint32_t taking_part = (uint32_t)__ballot(there);   // of lanes 0..31, a bit per token
#pragma unroll 1
      for (uint32_t n = 0; n < kTile; ++n) {
        if (!(taking_part >> n & 1)) continue;
        const char* value = values + __shfl(at, n);
        const float weight = __shfl(p, n);
#pragma unroll
        for (uint32_t i = 0; i < kOwn; ++i) {
          const uint32_t d = lane + 64 * i < D ? lane + 64 * i : 0;
          sum[i] = fmaf(weight, INT8 ? (float)((const int8_t*)value)[d] : bf16_value(((const uint16_t*)value)[d]), sum[i]);
        }
      }
    }
#pragma unroll
    for (uint32_t i = 0; i < kOwn; ++i)
      if (lane + 64 * i < D) lds_sum[(wave * kHeads + h) * (DIM + 4) + lane + 64 * i] = sum[i];
    if (lane == 0) lds_max[wave * kHeads + h] = m, lds_total[wave * kHeads + h] = sum_p;
  }
}

// Bound: reading the cache.  16 x 32768 tokens, 8 heads of 64 in bf16: 170..176 us, 6.1..6.3 TB/s; 1 x 131072 of 128: 87..92, 5.8..6.2; in 8 bits
// 16 x 32768 of 128: 174..190, 5.8..6.4, with the vector units busy nearly all of the time (conversion to bf16); 4 x 32768, 4 heads of 256: 93, 5.8.
// Few tokens: launch, lengths, page table, keys and values, join, 6.0 us for 200 tokens.
//
// All (row, chunk, unit of kUnit tokens) in this order are one line, cut into equal shares, one per workgroup: whatever the lengths, every
// workgroup has as much to do.  Eight wavefronts (one workgroup per compute unit) hold as much on its way as the memory needs: twelve and
// sixteen, or two workgroups per unit, leave too few registers for a tile ahead (16 x 16384 of 128: 188, 198, 281, 191 us).  A (row, chunk)
// that lies in one share is finished there; of one that is cut every workgroup leaves its maximum, total and weighted sum in memory and
// counts itself in, and the last one joins them, in the order of the line; more than kCluster parts are joined by clusters first.  Nobody
// waits for anybody.
//
// A wavefront asks for the next tile's keys as soon as the logits of this one are made, and for its values when they are multiplied
// in, also where the next tile is another row's: a row's end is worked on while the next one's first tile is on its way.  All of
// them are requested without a condition, keys ahead of values, and nothing else that is loaded is left unused: only then do the
// compiler's waits count the loads behind those they are for.  (In place of a tile that is not there all lanes read one word of
// the last one, and a page that is not there is read as page 0 and masked.)
template <int DIM, bool INT8, bool TRACK, bool PASSES>
__global__ __launch_bounds__(kAttendThreads, 2) void k_attend(CacheView c, AttendView a) {
  using T = Tile<DIM, INT8>;
  __shared__ __attribute__((aligned(16))) float lds_sum[kAttendWaves * kHeads * (DIM + 4)];   // [wave][head][DIM + 4]: heads in other banks
  __shared__ bf16x8 lds_q[T::kSteps][2][64];                // [step][0]: upper (columns 0..7) and middle 8 bits of q, [1]: lower ones, beside zeros
  __shared__ float lds_max[kAttendWaves * kHeads], lds_total[kAttendWaves * kHeads];            // [wave or group][head]
  __shared__ uint32_t lds_before;
  const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane / 16, n = lane % 16, head = n % 8, part = n / 8;
  const uint32_t D = c.head_dim, per_kv = a.chunks / c.kv_heads;
  auto scalar = [](uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); };

  // this workgroup's share, and the row it begins in
  uint32_t lane_length = 0, lane_seq = 0;   // of row (r & ~63) + lane
  auto look_at = [&](uint32_t first) {
    if (first + lane < a.rows) lane_length = row_length(c, a, first + lane, &lane_seq);
    return wave_prefix_sum(first + lane < a.rows ? units_of(lane_length) : 0u);
  };
  uint32_t upto = 0, all = 0, longest = 0;   // longest: units of a row
  for (uint32_t first = (a.rows - 1) & ~63u;; first -= 64) {   // (the first rows last: they stay in the lanes)
    upto = look_at(first);
    all += scalar(__shfl(upto, 63));
    longest = max(longest, units_of((uint32_t)__builtin_amdgcn_readlane((int)max_of_lanes(first + lane < a.rows ? lane_length : 0u), 63)));
    if (first == 0) break;
  }
  all *= a.chunks;
  const uint32_t even = (all + gridDim.x - 1) / gridDim.x;
  uint32_t share = even, quantum = 1;
  // Where the shares are small, a share that has the end of one row and the start of another is joined twice, one after the other, and a row
  // is in more parts than it need be.  So every (row, chunk) is rounded up to whole quanta, and a share is whole quanta: the longest row's
  // units, and no row is cut, or the fewest from an even share on with which every part has a workgroup.  Cut anywhere and so, us: 16 x 700
  // tokens of 64 dims 14.5 and 11.2, of 128 20.1 and 18.0; 16 x 1250 17.5 and 14.7, 25.9 and 22.4; 2 x 20000 23.0 and 20.9, 35.7 and 33.4; 16
  // ragged rows up to 2000 17.3 and 15.2, 24.2 and 22.1; but 12 x 2200 of 128 28.6 and 30.0.
  // Shares may be longer than even ones for that, since a compute unit alone draws 41 bytes per ns, among all of them 24, and a join takes
  // about 4 us: by a half up to four units (in 8 bits, 128 dims, 16 ragged rows up to 1500 17.1, by a quarter 18.6; up to 2500 20.5, 21.8),
  // by a quarter beyond (16 ragged rows up to 6000 43.4, by a half 47.4; 12 x 7000 of 64 dims 38, 42, of 128 64.5, 72).
  // A row of a few units is better not cut at all, the fewer bytes its tokens have: up to four units of keys of 64 bytes (16 x 1000 of 32
  // dims 10.8, cut 12.3; of 64 in 8 bits 12.0, 12.4; but of 64 in 16 bits 13.4, 12.5, of 128 22.8, 18.2), three of all others (16 x 700 of 64
  // dims 11.2, 12.2; of 96 15.1, 15.6; of 128 18.0, 17.5).  Where there is a workgroup for every unit, two units of up to 128 bytes (4 x 500
  // of 64 dims 8.0, cut 8.6, in 8 bits 8.2, 8.8; of 128 12.8, 11.5).
  // Shares of more than kMostAligned units take their next row's loads while they join, and are cut anywhere.
  constexpr uint32_t kMostBytes = (INT8 ? 1 : 2) * DIM;   // (of a key of this variant: a rule on D would cost the others 0.3 us)
  if (a.rows <= 64 && even <= kMostAligned && longest > 1 && (even > 1 || (longest == 2 && kMostBytes <= 128))) {
    const uint32_t units = lane < a.rows ? units_of(lane_length) : 0;
    auto attempt = [&](uint32_t q, uint32_t most) {
      const uint32_t quanta = wave_prefix_sum((uint32_t)(((float)(units + q - 1) + 0.5f) * __builtin_amdgcn_rcpf((float)q)));   // (exact: far fewer than 2^20 units)
      const uint32_t total = scalar(__shfl(quanta, 63)) * a.chunks, mine = total <= gridDim.x ? q : (total + gridDim.x - 1) / gridDim.x * q;
      if (mine > most) return false;
      upto = quanta * q, all = total * q, share = mine, quantum = q;
      return true;
    };
    bool done = longest <= (DIM <= 64 && (INT8 ? 1 : 2) * D <= 64 ? 4 : 3) && attempt(longest, even + (even > 1 ? 2 : 1));
    const uint32_t most = even + (even > 4 ? even / 4 : even / 2);
    for (uint32_t q = even; q <= most && !done; ++q) done = attempt(q, most);
  }
  uint32_t pos = blockIdx.x * share;
  uint32_t stop = min(pos + share, all);
  if (pos >= stop) return;
  uint32_t r = 0, row_first = 0;
  while (r < a.rows) {   // (all > pos: the row is found)
    const uint64_t beyond = __ballot(row_first + upto * a.chunks > pos);
    if (beyond) {
      const uint32_t at = (uint32_t)__builtin_ctzll(beyond);
      r += at;
      if (at) row_first += scalar(__shfl(upto, at - 1)) * a.chunks;
      break;
    }
    row_first += scalar(__shfl(upto, 63)) * a.chunks;
    r += 64;
    upto = look_at(r);
  }
  if (r >= a.rows) return;   // (lengths that change under the call)

  // a lane's places in a block of 16 tokens: for dims that a head does not have all lanes read the block's first ones, against zeros of q,
  // and drop them. With 256 dims of bf16 the tiles alone take 192 registers of the 256, and what spills waits for all that is on its way:
  // there one offset serves all loads of keys (where a head ends before a load's dims, it has the head's last ones once more), and the two
  // halves of the columns fetch half of q each (4 x 32768 tokens through the L2s: 110 -> 99 us).  Elsewhere that only adds to a call's start,
  // 0.1 to 0.5 us of 6 or 7.
  constexpr bool kTight = DIM == 256 && !INT8;
  constexpr uint32_t kSize = INT8 ? 1 : 2, kSpan = INT8 ? 64 : 32, kOffsets = kTight ? 1 : T::kLoads, kFetched = kTight ? 4 : 8;
  const uint32_t slot_bytes = kSize * (uint32_t)c.slot_stride;
  auto first_dim = [&](uint32_t s) { return !kTight ? kSpan * s : D >= kSpan ? min(kSpan * s, D - kSpan) : 0u; };
  uint32_t key_at[kOffsets];
#pragma unroll
  for (uint32_t s = 0; s < kOffsets; ++s) key_at[s] = kSpan * kSize * s + 16 * g < kSize * D ? n * slot_bytes + kSpan * kSize * s + 16 * g : 0;
  // A lane's dims of a value are neighbours.  Where they are two loads that pass the caches, each has eight neighbours and the second those
  // of the head's last 128: two from the same lines would read these twice.
  constexpr bool kApart = PASSES && T::kValWords > 4;
  constexpr uint32_t kNear = kApart ? T::kVals / 2 : T::kVals;
  const uint32_t val_at = n * kNear < D ? 4 * g * slot_bytes + kSize * n * kNear : 0, second_at = kSize * (D - 128);

  auto next_segment = [&] {
    Segment s;
    s.r = r;
    const uint32_t length = (uint32_t)__builtin_amdgcn_readlane((int)lane_length, r & 63);
    s.seq = (uint32_t)__builtin_amdgcn_readlane((int)lane_seq, r & 63);
    const uint32_t units = units_of(length);
    s.units = quantum == 1 ? units : (uint32_t)(((float)(units + quantum - 1) + 0.5f) * __builtin_amdgcn_rcpf((float)quantum)) * quantum;
    const uint32_t pair = (pos - row_first) / s.units;
    s.pair_first = row_first + pair * s.units;
    s.kv = pair / per_kv;
    const uint32_t chunk = pair % per_kv, unit = pos - s.pair_first, unit_end = min(s.units, unit + (stop - pos));
    s.first_head = s.kv * a.group + chunk * kHeads;
    s.n_heads = min((uint32_t)kHeads, a.group - chunk * kHeads);
    s.begin = unit * kUnit;
    s.end = min(length, unit_end * kUnit);
    s.rounds = min(unit_end, units) - unit;
    pos += unit_end - unit;
    if (pos == row_first + s.units * a.chunks) {
      row_first = pos;
      if (++r >= a.rows) stop = pos;
      else if ((r & 63) == 0 && pos < stop) look_at(r);
    }
    return s;
  };
  struct Blocks {   // two blocks of 16 tokens: their first byte in a pool, their first scale, how many tokens take part
    uint64_t at[2], mark[2];
    uint32_t limit[2];
  };
  auto blocks_of = [&](const Segment& s, uint32_t round) {
    constant_i32* table = (constant_i32*)(c.tables + (uint64_t)s.seq * c.table_stride);
    const uint32_t tile = s.begin + round * kUnit + wave * kTile, newest = max(s.end, 1u) - 1, there = min(tile, newest & ~(kTile - 1u));
    Blocks w;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const uint32_t at = there + 16 * b, want = tile + 16 * b, id = (uint32_t)table[min(at, newest) >> c.page_shift];
      w.limit[b] = id < c.n_pages && want < s.end ? min(s.end - want, 16u) : 0u;
      const uint32_t page = id < c.n_pages ? id : 0, slot = at & ((1u << c.page_shift) - 1);
      w.at[b] = kSize * ((uint64_t)page * c.page_stride + s.kv * c.head_stride + slot * c.slot_stride);
      w.mark[b] = INT8 ? (((uint64_t)page * c.kv_heads + s.kv) << c.page_shift) + slot : 0;
    }
    return w;
  };
  // (kept from being widened ahead of the loop: a 32-bit offset beside a scalar base takes one register and no addition)
  auto offset_of = [](uint32_t v) {
    asm("" : "+v"(v));
    return v;
  };
  T x;
  auto fetch_keys = [&](const Blocks& w) {   // (of a block without tokens all lanes read the same words)
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const char* from = c.k + w.at[b];
      const uint32_t lanes = w.limit[b] ? ~0u : 0u;
#pragma unroll
      for (int s = 0; s < T::kLoads; ++s) load_words<4, PASSES>(&x.k[b][4 * s], from + (kTight ? kSize * first_dim(s) : 0) + offset_of(key_at[kTight ? 0 : s] & lanes));
      if constexpr (INT8) x.ks[b] = *(const float4*)(c.k_scale + w.mark[b] + 4 * g);
    }
  };
  auto fetch_values = [&](const Blocks& w) {
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const uint32_t lanes = w.limit[b] ? ~0u : 0u;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const char* from = c.v + w.at[b] + j * slot_bytes;
        load_words<kApart ? 4 : T::kValWords, PASSES>(x.v[4 * b + j], from + offset_of(val_at & lanes));
        if constexpr (kApart) load_words<4, PASSES>(x.v[4 * b + j] + 4, from + second_at + offset_of(val_at & lanes));
      }
      if constexpr (INT8) x.vs[b] = *(const float4*)(c.v_scale + w.mark[b] + 4 * g);
    }
  };
  // 8 values of a segment's q: lane threadIdx.x % 64 of contraction step threadIdx.x / 64.  They are requested as words, two bf16 values in each,
  // from any address of their type and without a condition, so that nothing waits for them here (a lane without values reads the first ones).
  const uint32_t q_load = INT8 ? wave / 2 : wave, q_dim = first_dim(q_load) + (INT8 ? 16 * g + 8 * (wave % 2) : 8 * g), q_size = a.q16 ? 2 : 4;
  const bool has_q = q_dim >= kSpan * q_load && q_dim < D;
  constexpr uint32_t kHalf = kFetched / 2;   // words of bf16 values, which come twice
  uint32_t q_words[kFetched];
  auto fetch_q = [&](const Segment& s) {
    const uint64_t row = (uint64_t)a.q + q_size * (s.r * a.q_stride + s.first_head * D);
    const uint32_t lane_at = head < s.n_heads && has_q ? q_size * (head * D + q_dim + (kTight ? 4 * part : 0)) : 0;
#pragma unroll
    for (uint32_t j = 0; j < kFetched; ++j) q_words[j] = *(global_cu32_any*)(row + (a.q16 ? 0 : j / kHalf * 4 * kHalf) + 4 * (j % kHalf) + lane_at);
  };
  Segment s = next_segment();
  fetch_q(s);
  Blocks now = blocks_of(s, 0);
  __builtin_amdgcn_sched_barrier(0);   // keys ahead of values, here too: the waits in the loop go by the worst order there is
  fetch_keys(now);
  __builtin_amdgcn_sched_barrier(0);
  fetch_values(now);
  __builtin_amdgcn_sched_barrier(0);
  for (;;) {
    static_assert(T::kSteps <= kAttendWaves, "a wavefront per step of q");
    bf16x8 q0, q1;
#pragma unroll
    for (int j = 0; j < 8; ++j) {   // (by all wavefronts: a load that some of them never use would be waited for in the loop)
      const uint32_t own = a.q16 ? q_words[j % kFetched / 2] : q_words[j % kFetched], other = kTight ? ror8(own) : own, word = (j < 4) == (part == 0) ? own : other;
      const float one = __uint_as_float((word << (a.q16 && j % 2 == 0 ? 16 : 0)) & (a.q16 ? 0xFFFF0000u : ~0u));
      const float v = head < s.n_heads && has_q ? one * a.scale : 0.f;
      const __bf16 hi = (__bf16)v, mid = (__bf16)(v - (float)hi), lo = (__bf16)(v - (float)hi - (float)mid);
      q0[j] = part ? mid : hi;
      q1[j] = part ? (__bf16)0.f : lo;
    }
    if (wave < T::kSteps) lds_q[wave][0][lane] = q0, lds_q[wave][1][lane] = q1;
    __syncthreads();

    f32x4 o[T::kVals];
#pragma unroll
    for (int b = 0; b < T::kVals; ++b) o[b] = f32x4{0.f, 0.f, 0.f, 0.f};
    float top = -INFINITY, total = 0.f;
    const bool more = pos < stop;
    Segment next_s = s;
#pragma clang loop unroll(disable)   // (nor peeled: the copies between the two forms would wait for what is on its way)
    for (uint32_t round = 0;; ++round) {
      const bool last = round + 1 == s.rounds;
      if (last && more) {
        next_s = next_segment();
        fetch_q(next_s);
      }
      Blocks next = now;
      next.limit[0] = next.limit[1] = 0;
      if (!last || more) next = blocks_of(next_s, last ? 0 : round + 1);
      asm volatile("" ::: "memory");   // q is read from LDS for every tile: registers are for what is on its way
      f32x4 l[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
      for (int s = 0; s < T::kSteps; ++s) {
        const bf16x8 q0 = lds_q[s][0][lane], q1 = lds_q[s][1][lane];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          bf16x8 key;
          if constexpr (INT8) key = i8x8_to_bf16x8(make_uint2(x.k[b][2 * s], x.k[b][2 * s + 1]));
          else key = __builtin_bit_cast(bf16x8, make_uint4(x.k[b][4 * s], x.k[b][4 * s + 1], x.k[b][4 * s + 2], x.k[b][4 * s + 3]));
          l[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(key, q0, l[b], 0, 0, 0);
          l[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(key, q1, l[b], 0, 0, 0);
        }
      }
      float p[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        p[i] = ror8_sum(l[i / 4][i % 4]);
        if constexpr (INT8) p[i] *= (&x.ks[i / 4].x)[i % 4];
      }
      __builtin_amdgcn_sched_barrier(0);
      fetch_keys(next);
      __builtin_amdgcn_sched_barrier(0);
      // Tokens that take no part: their weight is 0, and the bits of their values are masked out, whatever lies there.  (The masks, and not the
      // loaded words, are what the branch changes: a word that it changed would be waited for there.)
      uint32_t value_bits[4] = {~0u, ~0u, ~0u, ~0u};   // of two neighbouring tokens
      if (now.limit[0] < 16 || now.limit[1] < 16) {
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
          const uint32_t at = 4 * g + i % 4, limit = now.limit[i / 4];
          if (at >= limit) p[i] = -INFINITY;
          if (at + 1 >= limit) p[i + 1] = -INFINITY;
          value_bits[i / 2] = at >= limit ? 0u : at + 1 >= limit ? 0xFFFFu : ~0u;
        }
      }
      if constexpr (TRACK) {
        // Both halves of the columns hold the same logits: one stores the first block, the other the second.  Lanes without a head or
        // a token store beyond the buffer's end, which drops it: no branch, so that the waits below still count.
        const uint32_t t = s.begin + round * kUnit + wave * kTile;
        const bool stores = head < s.n_heads && t + 16 * part < s.end;
        float* to = a.logits + ((uint64_t)s.r * a.heads + s.first_head) * c.capacity + t;
        const auto rows = __builtin_amdgcn_make_buffer_rsrc(to, 0, 0x7FFFFFFF, 0x00020000);
        const u32x4 four = {__float_as_uint(part ? p[4] : p[0]), __float_as_uint(part ? p[5] : p[1]), __float_as_uint(part ? p[6] : p[2]), __float_as_uint(part ? p[7] : p[3])};
        __builtin_amdgcn_raw_buffer_store_b128(four, rows, stores ? (int)(4 * (head * c.capacity + 16 * part + 4 * g)) : -16, 0, 0);
      }
      float m = top;
#pragma unroll
      for (int i = 0; i < 8; ++i) m = fmaxf(m, p[i]);
      m = fmaxf(m, __shfl_xor(m, 16));
      m = fmaxf(m, __shfl_xor(m, 32));
      const float base = m == -INFINITY ? 0.f : m;   // nothing here takes part
      const float shrink = __builtin_amdgcn_exp2f(top - base);
      top = m;
      total *= shrink;
#pragma unroll
      for (int b = 0; b < T::kVals; ++b) o[b] *= shrink;
      uint32_t p0[4], p1[4];   // pairs of tokens
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        float w[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          w[j] = __builtin_amdgcn_exp2f(p[i + j] - base);
          total += w[j];
          if constexpr (INT8) w[j] = p[i + j] != -INFINITY ? w[j] * (&x.vs[i / 4].x)[i % 4 + j] : 0.f;   // (a masked token's scale may be anything)
        }
        const uint32_t hi = pack_bf16(w[0], w[1]);
        w[0] -= bf16_value(hi), w[1] -= __uint_as_float(hi & 0xFFFF0000u);
        const uint32_t mid = pack_bf16(w[0], w[1]);
        w[0] -= bf16_value(mid), w[1] -= __uint_as_float(mid & 0xFFFF0000u);
        p0[i / 2] = part ? mid : hi, p1[i / 2] = part ? 0 : pack_bf16(w[0], w[1]);
      }
      const bf16x8 upper = __builtin_bit_cast(bf16x8, make_uint4(p0[0], p0[1], p0[2], p0[3])), lower = __builtin_bit_cast(bf16x8, make_uint4(p1[0], p1[1], p1[2], p1[3]));
#pragma unroll
      for (int b = 0; b < T::kVals; ++b) {
        uint32_t vt[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if constexpr (INT8) {
            const float lo = (float)(int8_t)(x.v[2 * i][b / 4] >> (8 * (b % 4))), hi = (float)(int8_t)(x.v[2 * i + 1][b / 4] >> (8 * (b % 4)));
            vt[i] = __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);   // (finite, so that a weight of 0 is enough)
          } else {
            vt[i] = __builtin_amdgcn_perm(x.v[2 * i + 1][b / 2], x.v[2 * i][b / 2], b % 2 ? 0x07060302u : 0x05040100u) & value_bits[i];
          }
        }
        const bf16x8 value = __builtin_bit_cast(bf16x8, make_uint4(vt[0], vt[1], vt[2], vt[3]));
        o[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(value, upper, o[b], 0, 0, 0);
        o[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(value, lower, o[b], 0, 0, 0);
        if constexpr (INT8) asm volatile("" : "+v"(o[b]));   // (values are widened as they are needed: all of them ahead, 256 dims spill 47 registers, 54 -> 70 us)
      }
      __builtin_amdgcn_sched_barrier(0);
      fetch_values(next);
      __builtin_amdgcn_sched_barrier(0);
      now = next;
      if (last) break;
    }

    // join the wavefronts: lane (g, head) holds dims (4 g + j) * kNear + b of the head, halves of p beside each other.  (Places in LDS and memory are
    // made here from the thread's number, which looks new each time: made ahead of all loops they take registers from the tiles, and with 256 dims of
    // bf16 come back from memory behind the next row's tile, 4 x 32768 tokens 106 us in place of 93.)
    uint32_t thread = threadIdx.x;
    asm volatile("" : "+v"(thread));
    const uint32_t lane = thread & 63, g = lane / 16, head = lane % 8, part = lane / 8 % 2;
    total += __shfl_xor(total, 16);
    total += __shfl_xor(total, 32);
    if (lane < kHeads) lds_max[wave * kHeads + lane] = top, lds_total[wave * kHeads + lane] = total;
#pragma unroll
    for (int b = 0; b < T::kVals; b += 4)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float4 v = make_float4(ror8_sum(o[b][j]), ror8_sum(o[b + 1][j]), ror8_sum(o[b + 2][j]), ror8_sum(o[b + 3][j]));
        if (part == 0) *(float4*)&lds_sum[(wave * kHeads + head) * (DIM + 4) + (b < (int)kNear ? 0 : D - 128) + (4 * g + j) * kNear + b % kNear] = v;
      }
    // A query, key or value that is not finite has met zeros and parts of opposite sign: no total or sum that it went into is finite.
    float odd = total * 0.f;
#pragma unroll
    for (int b = 0; b < T::kVals; ++b)
#pragma unroll
      for (int j = 0; j < 4; ++j) odd = fmaf(o[b][j], 0.f, odd);
    if (__builtin_expect(__any(!(odd == 0.f)), 0)) take_again<DIM, INT8, TRACK>(s, lane, wave, lds_sum, lds_max, lds_total);
    __syncthreads();
    // the workgroups among which this (row, chunk) is cut
    const uint32_t n_heads = s.n_heads, group0 = s.pair_first / share, parts = min((s.pair_first + s.units - 1) / share, gridDim.x - 1) - group0 + 1;
    const uint64_t slot_floats = kHeads * (D + 2);
    auto slot_of = [&](uint32_t group) { return a.partials + (2 * (uint64_t)group + (group * share >= s.pair_first ? 0 : 1)) * slot_floats; };
    // a group of DIM / 4 lanes per head, four dims a lane
    constexpr uint32_t kLanes = DIM / 4, kGroups = kAttendThreads / kLanes;
    static_assert(kGroups >= kHeads && kGroups <= kAttendWaves * kHeads, "a group per head; lds_max");
    const uint32_t of_group = thread / kLanes, d0 = thread % kLanes * 4;
    const bool joins = of_group < n_heads && d0 < D;
    struct Joined {
      float4 sum;
      float m, sum_p;
    };
    auto joined = [&](uint32_t n, uint32_t heads_n) {   // n parts in LDS, [part][heads_n][DIM + 4] -> the whole
      Joined j = {make_float4(0.f, 0.f, 0.f, 0.f), -INFINITY, 0.f};
#pragma unroll 4
      for (uint32_t w = 0; w < n; ++w) j.m = fmaxf(j.m, lds_max[w * heads_n + of_group]);
      const float base = j.m == -INFINITY ? 0.f : j.m;
#pragma unroll 4
      for (uint32_t w = 0; w < n; ++w) {
        const float f = __builtin_amdgcn_exp2f(lds_max[w * heads_n + of_group] - base);
        const float4 v = *(const float4*)&lds_sum[(w * heads_n + of_group) * (DIM + 4) + d0];
        j.sum.x = fmaf(f, v.x, j.sum.x), j.sum.y = fmaf(f, v.y, j.sum.y), j.sum.z = fmaf(f, v.z, j.sum.z), j.sum.w = fmaf(f, v.w, j.sum.w);
        j.sum_p = fmaf(f, lds_total[w * heads_n + of_group], j.sum_p);
      }
      return j;
    };
    auto finish = [&](const Joined& j) {
      const float inv = j.sum_p == 0.f ? 0.f : 1.f / j.sum_p;
      uint16_t* to = a.out + s.r * a.out_stride + (s.first_head + of_group) * D + d0;
      const uint32_t lo = pack_bf16(j.sum.x * inv, j.sum.y * inv), hi = pack_bf16(j.sum.z * inv, j.sum.w * inv);
      if (a.out_by4) *(uint2*)to = make_uint2(lo, hi);
      else to[0] = (uint16_t)lo, to[1] = (uint16_t)(lo >> 16), to[2] = (uint16_t)hi, to[3] = (uint16_t)(hi >> 16);
      if (TRACK && d0 == 0) a.stats[(uint64_t)s.r * a.heads + s.first_head + of_group] = make_float2(j.m == -INFINITY ? 0.f : j.m, inv);
    };
    if (parts == 1) {
      if (joins) finish(joined(kAttendWaves, kHeads));
    } else {
      typedef __attribute__((address_space(1))) uint32_t global_u32;
      typedef __attribute__((address_space(1))) uint64_t global_u64;
      // stored to and loaded from the level that the device shares (an acquire fence would empty an L2 that the others read through)
      auto left_by = [&](const float* p) {
        return __builtin_bit_cast(float2, __hip_atomic_load((global_u64*)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
      };
      auto leave = [&](float* p, float x, float y) {
        __hip_atomic_store((global_u64*)p, __builtin_bit_cast(uint64_t, make_float2(x, y)), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      };
      // what is joined first: this workgroup's wavefronts; then, if there are many parts, those of a cluster; then all, or the clusters'
      const uint32_t cluster = blockIdx.x / kCluster, last_group = group0 + parts - 1;
      bool whole = parts <= kCluster;
      uint32_t first_part = whole ? group0 : max(group0, cluster * kCluster), n = whole ? parts : min(last_group, cluster * kCluster + kCluster - 1) - first_part + 1;
      float* mine = slot_of(blockIdx.x);
      uint32_t in_lds = kAttendWaves, in_lds_heads = kHeads;
      for (;;) {
        if (joins) {
          const Joined j = joined(in_lds, in_lds_heads);
          if (n == 0) {
            finish(j);
          } else {
            leave(mine + of_group * D + d0, j.sum.x, j.sum.y);
            leave(mine + of_group * D + d0 + 2, j.sum.z, j.sum.w);
            if (d0 == 0) leave(mine + kHeads * D + 2 * of_group, j.m, j.sum_p);
          }
        }
        if (n == 0) break;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // the stores have reached the level that the device shares
        __syncthreads();
        // (a cluster has parts of at most two rows that reach beyond it: one that begins before it, one that begins in it)
        global_u32* arrived = (global_u32*)(whole ? a.arrived + 2 * (kMaxGroups / kCluster) + group0
                                                  : a.arrived + 2 * cluster + (group0 >= cluster * kCluster ? 1 : 0));
        if (thread == 0) lds_before = __hip_atomic_fetch_add(arrived, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __syncthreads();
        if (lds_before != n - 1) break;   // the last one joins: the others' parts are in
        if (thread == 0) __hip_atomic_store(arrived, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        // every group takes a head and every per_head-th part, kAhead parts at a time
        constexpr uint32_t kAhead = 4;
        const uint32_t heads_n = n_heads > 4 ? 8 : n_heads > 2 ? 4 : n_heads, per_head = kGroups / heads_n, h = of_group % heads_n, part0 = of_group / heads_n;
        const bool of_clusters = whole && parts > kCluster;
        if (h < n_heads) {
          float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
          float m = -INFINITY, sum_p = 0.f;
          for (uint32_t v = part0; v < n; v += kAhead * per_head) {
            float2 sums[kAhead][2], st[kAhead];
#pragma unroll
            for (uint32_t i = 0; i < kAhead; ++i) {
              const uint32_t w = min(v + i * per_head, n - 1);
              const float* from = slot_of(of_clusters ? max(group0, (group0 / kCluster + w) * kCluster) : first_part + w);
              const float* at = from + h * D + (d0 < D ? d0 : 0);
              sums[i][0] = left_by(at), sums[i][1] = left_by(at + 2);
              st[i] = left_by(from + kHeads * D + 2 * h);
            }
#pragma unroll
            for (uint32_t i = 0; i < kAhead; ++i) {
              if (v + i * per_head >= n) continue;
              const float to = fmaxf(m, st[i].x), base = to == -INFINITY ? 0.f : to;
              const float f = __builtin_amdgcn_exp2f(m - base), e = __builtin_amdgcn_exp2f(st[i].x - base);
              m = to;
              sum_p = sum_p * f + st[i].y * e;
              sum.x = sum.x * f + sums[i][0].x * e, sum.y = sum.y * f + sums[i][0].y * e;
              sum.z = sum.z * f + sums[i][1].x * e, sum.w = sum.w * f + sums[i][1].y * e;
            }
          }
          __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0): none of these loads is left for the loop to wait for
          if (d0 == 0) lds_max[of_group] = m, lds_total[of_group] = sum_p;
          *(float4*)&lds_sum[of_group * (DIM + 4) + d0] = sum;
        }
        __syncthreads();
        in_lds = per_head, in_lds_heads = heads_n;
        if (whole) {
          n = 0;
        } else {   // the cluster's parts become one, in the first one's place
          mine = slot_of(first_part);
          whole = true, n = last_group / kCluster - group0 / kCluster + 1;
        }
      }
    }
    if (!more) break;
    __syncthreads();   // LDS is free again
    s = next_s;
  }
}

// Adds the weights of all rows of a sequence to its slots' scores, rows and heads in order; four slots a thread.  Bound: a launch and, for long
// lists, reading the logits (8 x 8179 tokens of 32 heads, 8 MB: 4.9 us).
__global__ __launch_bounds__(256) void k_attend_scores(CacheView c, AttendView a) {
  const uint32_t slot = (blockIdx.x * 256 + threadIdx.x) * 4, kv = blockIdx.y, s = blockIdx.z;
  if (slot >= c.capacity) return;   // (a multiple of 16)
  float* to = c.scores + ((uint64_t)s * c.kv_heads + kv) * c.capacity + slot;
  const f32x4_any were = *(const f32x4_any*)to;
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
  int32_t longest = 0;
  const uint32_t r0 = a.seqs ? 0 : s, r1 = a.seqs ? a.rows : min(a.rows, s + 1);
  for (uint32_t r = r0; r < r1; ++r) {
    if (a.seqs && a.seqs[r] != (int32_t)s) continue;
    const int32_t length = a.lengths[r];
    if ((int64_t)slot >= (int64_t)length) continue;
    longest = max(longest, length);
#pragma unroll 4
    for (uint32_t h = kv * a.group; h < (kv + 1) * a.group; ++h) {
      const float2 st = a.stats[(uint64_t)r * a.heads + h];
      const float4 l = *(const float4*)(a.logits + ((uint64_t)r * a.heads + h) * c.capacity + slot);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if ((int64_t)slot + j < (int64_t)length) sum[j] += __builtin_amdgcn_exp2f((&l.x)[j] - st.x) * st.y;
    }
  }
  if ((int64_t)slot + 4 <= (int64_t)longest) {
    *(f32x4_any*)to = were + f32x4_any{sum[0], sum[1], sum[2], sum[3]};
  } else {
#pragma unroll
    for (int j = 0; j < 3; ++j)
      if ((int64_t)slot + j < (int64_t)longest) to[j] = were[j] + sum[j];
  }
}

struct Layout {
  uint64_t arrived, partials, logits, stats, bytes;   // offsets
  uint32_t chunks, groups;
};

int check_attend(const std::string& who, const tq_cache* cache, const tq_attend_args* a, CacheView* c, Layout* l) {
  if (int rc = view_cache(who, cache, c)) return rc;
  if (!a) return refuse(TQ_E_INVALID_ARG, who + ": null argument");
  if (a->q_type != TQ_FP32 && a->q_type != TQ_BF16) return refuse(TQ_E_UNSUPPORTED, who + ": q is TQ_FP32 or TQ_BF16");
  if (a->heads == 0 || a->heads > 65535 || a->heads % c->kv_heads) return refuse(TQ_E_INVALID_ARG, who + ": heads must be a multiple of kv_heads up to 65535");
  if (a->rows > 65535) return refuse(TQ_E_UNSUPPORTED, who + ": more than 65535 rows");
  if (!a->seqs && a->rows > c->n_seqs) return refuse(TQ_E_INVALID_ARG, who + ": more rows than sequences, and no seqs");
  if (a->accumulate > 1) return refuse(TQ_E_INVALID_ARG, who + ": accumulate is 0 or 1");
  if (a->accumulate && c->capacity > (1u << 25)) return refuse(TQ_E_UNSUPPORTED, who + ": accumulate needs a capacity of at most 2^25 tokens");
  if (a->accumulate && !c->scores) return refuse(TQ_E_INVALID_ARG, who + ": the cache has no scores to add to");
  if (!(a->scale > 0.f) || !(a->scale < INFINITY)) return refuse(TQ_E_INVALID_ARG, who + ": scale must be positive");
  const uint32_t group = a->heads / c->kv_heads;
  l->chunks = c->kv_heads * ((group + kHeads - 1) / kHeads);
  const uint64_t most = (uint64_t)a->rows * l->chunks * ((c->capacity + kUnit - 1) / kUnit);   // units, if all rows are full
  if (most >= (1u << 31) - kMaxGroups) return refuse(TQ_E_UNSUPPORTED, who + ": rows * heads * capacity is beyond what one call takes");
  l->groups = (uint32_t)std::min<uint64_t>(kMaxGroups, std::max<uint64_t>(1, most));
  auto place = [&](uint64_t n) {
    const uint64_t at = l->bytes;
    l->bytes += (n + 255) / 256 * 256;
    return at;
  };
  l->bytes = 0;
  l->arrived = place(kCounters * 4);   // first, and as many for every call
  l->partials = place((uint64_t)l->groups * 2 * kHeads * (c->head_dim + 2) * 4);
  l->logits = a->accumulate ? place((uint64_t)a->rows * a->heads * c->capacity * 4) : 0;
  l->stats = a->accumulate ? place((uint64_t)a->rows * a->heads * 8) : 0;
  return TQ_OK;
}

// passes: keys and values are not kept in the caches.
template <int DIM>
void launch_attend(const CacheView& c, const AttendView& a, uint32_t groups, bool int8, bool track, bool passes, hipStream_t stream) {
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(groups), dim3(kAttendThreads), 0, stream, c, a); };
  auto of = [&](auto eight) {
    constexpr bool I = decltype(eight)::value;
    if constexpr (kPasses<DIM, I>) {
      if (passes) return track ? go(k_attend<DIM, I, true, true>) : go(k_attend<DIM, I, false, true>);
    }
    track ? go(k_attend<DIM, I, true, false>) : go(k_attend<DIM, I, false, false>);
  };
  int8 ? of(std::true_type()) : of(std::false_type());
}

int attend(const tq_cache* cache, const tq_attend_args* a, void* stream) {
  const std::string who = "tq_attend";
  CacheView c;
  Layout l;
  if (int rc = check_attend(who, cache, a, &c, &l)) return rc;
  if (a->rows == 0) return TQ_OK;
  if (!a->q || !a->out || !a->lengths || !a->workspace) return refuse(TQ_E_INVALID_ARG, who + ": null pointer");
  const uint64_t row = (uint64_t)a->heads * c.head_dim;
  const bool q16 = a->q_type == TQ_BF16;
  if (!aligned_to(a->q, q16 ? 2 : 4) || !aligned_to(a->out, 2) || !aligned_to(a->seqs, 4) || !aligned_to(a->lengths, 4) || !aligned_to(a->workspace, 16))
    return refuse(TQ_E_INVALID_ARG, who + ": a pointer is not aligned to its type (workspace: 16 bytes)");
  if ((a->q_stride && a->q_stride < row) || (a->out_stride && a->out_stride < row)) return refuse(TQ_E_INVALID_ARG, who + ": a stride is smaller than a row");
  if (a->workspace_bytes < l.bytes)
    return refuse(TQ_E_INVALID_ARG, who + ": the workspace has " + std::to_string(a->workspace_bytes) + " bytes, " + std::to_string(l.bytes) + " are needed");
  char* ws = (char*)a->workspace;
  const AttendView v{a->q, (uint16_t*)a->out, a->seqs, a->lengths, (uint32_t*)(ws + l.arrived), (float*)(ws + l.partials), (float*)(ws + l.logits),
                     (float2*)(ws + l.stats), a->q_stride ? a->q_stride : row, a->out_stride ? a->out_stride : row,
                     a->scale * kLog2e, a->rows, a->heads, a->heads / c.kv_heads, l.chunks, q16,
                     (a->out_stride ? a->out_stride : row) % 4 == 0 && aligned_to(a->out, 8)};
  const bool int8 = cache->type == TQ_INT8;
  hipStream_t s = (hipStream_t)stream;
  // Little may still be in the L2s (200 tokens of 128 dims 7.5 us, passing them by 8.3; 8 x 1000 of 64 10.8 and 10.3), and what several rows of a
  // sequence or several chunks of query heads read shall stay there (32 heads on 2, 16 x 8000 tokens 44.5 and 50).  By the capacity, since only
  // the GPU knows the lengths.
  const uint64_t bytes = (uint64_t)a->rows * c.kv_heads * c.capacity * c.head_dim * (int8 ? 2 : 4);
  // (256 dims of bf16: 33 MB 19.2 us and 19.6, 66 MB 23.9 and 23.4; of 208, whose last 128 overlap the first, 4 x 8000 28.7 and 34.7.)
  const bool passes = !a->seqs && l.chunks == c.kv_heads && bytes >= (c.head_dim == 256 && !int8 ? 8 * kPassing : kPassing) &&
                      c.head_dim % 32 == 0 && c.head_dim >= (c.head_dim <= 128 ? 64 : int8 ? 192 : 256);
  if (c.head_dim <= 64) launch_attend<64>(c, v, l.groups, int8, a->accumulate, passes, s);
  else if (c.head_dim <= 128) launch_attend<128>(c, v, l.groups, int8, a->accumulate, passes, s);
  else launch_attend<256>(c, v, l.groups, int8, a->accumulate, passes, s);
  if (a->accumulate) hipLaunchKernelGGL(k_attend_scores, dim3((c.capacity + 1023) / 1024, c.kv_heads, c.n_seqs), dim3(256), 0, s, c, v);
  return launched("tq_attend");
}

}  // namespace
}  // namespace tq

extern "C" int tq_attend(const tq_cache* cache, const tq_attend_args* args, void* stream) {
  return tq::contained("tq_attend", [&] { return tq::attend(cache, args, stream); });
}

extern "C" int tq_attend_workspace(const tq_cache* cache, const tq_attend_args* args, uint64_t* bytes) {
  return tq::contained("tq_attend_workspace", [&] {
    if (!bytes) return tq::refuse(TQ_E_INVALID_ARG, "tq_attend_workspace: null argument");
    tq::CacheView c;
    tq::Layout l;
    const int rc = tq::check_attend("tq_attend_workspace", cache, args, &c, &l);
    if (rc == TQ_OK) *bytes = l.bytes;
    return rc;
  });
}
