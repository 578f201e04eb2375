// Attention of one new token per row over a paged cache (tq_attend).
//
// A wavefront takes 32 tokens of one key/value head at a time and up to 8 of the query heads that share it.  Both products run on
// v_mfma_f32_16x16x32_bf16, keys and values go from memory to registers in the shape the instruction wants, and nothing passes
// through LDS or between lanes but the softmax maxima:
//   logits^T [token][head] = K [token][dim] Q^T: lane l supplies token l % 16 and 8 neighbouring dims (16 bytes of a key).
//   out^T [dim][head] = V^T [dim][token] P^T: the lane that got the logits of tokens 4g..4g+3 of both 16-token blocks (g = l / 16)
//   supplies the same tokens as its 8 values of the contraction, so P is already where it is needed; it loads DIM / 16
//   neighbouring dims of those 8 tokens' values and transposes that square in its registers (one v_perm per pair).
// The 16 columns are 8 heads twice: column c holds the upper 8 bits of head c's mantissas, column c + 8 the next 8, so that
// q (three parts, two products) enters with all of fp32's 24 bits and p with 16, at a few per cent of the matrix unit's rate.
#include <algorithm>

#include "tq_cache_view.h"
#include "tq_strip_decode.h"

namespace tq {
namespace {

constexpr int kAttendWaves = 4, kAttendThreads = kAttendWaves * 64, kTile = 32, kHeads = 8;   // kHeads: query heads of a workgroup
constexpr uint32_t kUnit = kAttendWaves * kTile;                          // tokens that a workgroup takes at a time
constexpr uint32_t kMaxGroups = 512, kMinShare = 2;                       // workgroups of a launch; units of one
constexpr float kLog2e = 1.4426950408889634f;

struct AttendView {
  const void* q;
  uint16_t* out;
  const int32_t *seqs, *lengths;
  uint32_t* arrived;   // [row][chunk]: workgroups whose part is in the partials; zero between calls
  float* partials;     // [workgroup][2]: kHeads x head_dim sums, then maximum and total of every head
  float* logits;       // [row][head][capacity], in units of log 2 (accumulate)
  float2* stats;       // [row][head]: maximum and 1 / total of the whole row (accumulate)
  uint64_t q_stride, out_stride;
  float scale;         // times log2(e)
  uint32_t rows, heads, group, chunks, q16;   // chunks: of up to kHeads query heads that share a key/value head, of all of these
};

__device__ __forceinline__ float ror8_sum(float v) {   // v of this lane + v of the lane 8 columns on
  return v + __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), 0x128, 0xf, 0xf, true));
}

__device__ __forceinline__ uint32_t row_length(const CacheView& c, const AttendView& a, uint32_t r, uint32_t* seq) {
  const int32_t s = a.seqs ? a.seqs[r] : (int32_t)r;
  *seq = (uint32_t)s < c.n_seqs ? (uint32_t)s : 0;
  return (uint32_t)s < c.n_seqs ? (uint32_t)min(max(a.lengths[r], 0), (int32_t)c.capacity) : 0;
}

typedef __attribute__((address_space(4))) const int32_t constant_i32;

template <int DIM, bool INT8>
struct Tile {
  static constexpr int kSteps = DIM / 32, kVals = DIM / 16;   // contraction steps of the logits; a lane's dims of a value
  static constexpr int kKeyWords = INT8 ? kSteps * 2 : kSteps * 4, kValWords = INT8 ? kVals / 4 : kVals / 2;
  uint32_t k[2][kKeyWords], v[8][kValWords];
  float4 ks[2], vs[2];
  uint32_t limit[2];   // tokens of a 16-token block that take part
};

template <int WORDS>
__device__ __forceinline__ void load_words(uint32_t* to, const char* from) {
  if constexpr (WORDS % 4 == 0) {
#pragma unroll
    for (int w = 0; w < WORDS; w += 4) {
      const uint4 d = *(const uint4*)(from + 4 * w);
      to[w] = d.x, to[w + 1] = d.y, to[w + 2] = d.z, to[w + 3] = d.w;
    }
  } else if constexpr (WORDS == 2) {
    const uint2 d = *(const uint2*)from;
    to[0] = d.x, to[1] = d.y;
  } else {
    to[0] = *(const uint32_t*)from;
  }
}

__device__ __forceinline__ uint32_t units_of(uint32_t length) { return max((length + kUnit - 1) / kUnit, 1u); }   // (an empty row is written too)

// Adds a wavefront-uniform running sum up over 64 lanes: inclusive prefix sums.
__device__ __forceinline__ uint32_t prefix_sum(uint32_t v) {
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xf, 0xf, true);
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xf, 0xf, true);
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xf, 0xf, true);
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xf, 0xf, true);
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xa, 0xf, false);   // lane 15 of a row to the next one
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xc, 0xf, false);   // lane 31 to the upper half
  return v;
}

// All (row, chunk, unit of kUnit tokens) in this order are one line, cut into equal shares, one per workgroup: whatever the
// lengths, every workgroup has as much to do.  A (row, chunk) that lies in one share is finished there; of one that is cut every
// workgroup leaves its maximum, total and weighted sum in memory and counts itself in, and the last one joins them, in the order
// of the line.  Nobody waits for anybody.
//
// A wavefront always has the next tile's loads on their way while it works on one: they are requested without a condition, so
// that the wait for a tile counts the loads behind it (the last tile is requested again in place of one that is not there, and a page
// that is not there is read as page 0 and masked).
template <int DIM, bool INT8, bool TRACK>
__global__ __launch_bounds__(kAttendThreads, DIM == 256 ? 1 : 2) void k_attend(CacheView c, AttendView a) {
  using T = Tile<DIM, INT8>;
  __shared__ __attribute__((aligned(16))) float lds_sum[kAttendWaves * kHeads * (DIM + 4)];   // [wave][head][DIM + 4]: heads in other banks
  __shared__ float lds_max[16 * kHeads], lds_total[16 * kHeads];                        // [wave or group][head]
  __shared__ uint32_t lds_before;
  const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane / 16, n = lane % 16, head = n % 8, part = n / 8;
  const uint32_t D = c.head_dim, per_kv = a.chunks / c.kv_heads;
  auto scalar = [](uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); };

  // this workgroup's share, and the row it begins in
  auto row_units = [&](uint32_t r) {
    uint32_t seq;
    return r < a.rows ? units_of(row_length(c, a, r, &seq)) : 0u;
  };
  uint32_t all = 0;
  for (uint32_t r = 0; r < a.rows; r += 64) all += scalar(__shfl(prefix_sum(row_units(r + lane)), 63));
  all *= a.chunks;
  const uint32_t share = max(kMinShare, (all + gridDim.x - 1) / gridDim.x);
  uint32_t pos = blockIdx.x * share;
  const uint32_t stop = min(pos + share, all);
  if (pos >= stop) return;
  uint32_t r = 0, row_first = 0;
  for (uint32_t base = 0;; base += 64) {   // (all > pos: the row is found)
    const uint32_t upto = prefix_sum(row_units(base + lane));
    const uint64_t beyond = __ballot(row_first + upto * a.chunks > pos);
    if (beyond) {
      const uint32_t at = (uint32_t)__builtin_ctzll(beyond);
      r = base + at;
      if (at) row_first += scalar(__shfl(upto, at - 1)) * a.chunks;
      break;
    }
    row_first += scalar(__shfl(upto, 63)) * a.chunks;
  }

  while (pos < stop) {
  uint32_t seq;
  const uint32_t length = scalar(row_length(c, a, r, &seq)), units = units_of(length);
  seq = scalar(seq);
  const uint32_t pair = (pos - row_first) / units, unit = (pos - row_first) % units, unit_end = min(units, unit + (stop - pos));
  const uint32_t kv = pair / per_kv, chunk = pair % per_kv;
  const uint32_t begin = unit * kUnit, end = min(length, unit_end * kUnit);
  const uint32_t first_head = kv * a.group + chunk * kHeads, n_heads = min((uint32_t)kHeads, a.group - chunk * kHeads);
  constant_i32* table = (constant_i32*)(c.tables + (uint64_t)seq * c.table_stride);

  // the query's parts: [step][0]: upper (columns 0..7) and middle 8 bits, [1]: lower ones, beside zeros
  bf16x8 q[T::kSteps][2];
#pragma unroll
  for (int s = 0; s < T::kSteps; ++s) {
    const uint32_t d0 = INT8 ? 64 * (s / 2) + 16 * g + 8 * (s % 2) : 32 * s + 8 * g;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float x = 0.f;
      if (head < n_heads && d0 < D) {
        const uint64_t at = r * a.q_stride + (first_head + head) * D + d0 + j;
        x = (a.q16 ? bf16_value(((const uint16_t*)a.q)[at]) : ((const float*)a.q)[at]) * a.scale;
      }
      const __bf16 hi = (__bf16)x, mid = (__bf16)(x - (float)hi), lo = (__bf16)(x - (float)hi - (float)mid);
      q[s][0][j] = part ? mid : hi;
      q[s][1][j] = part ? (__bf16)0.f : lo;
    }
  }

  f32x4 o[T::kVals];
#pragma unroll
  for (int b = 0; b < T::kVals; ++b) o[b] = f32x4{0.f, 0.f, 0.f, 0.f};
  float top = -INFINITY, total = 0.f;

  struct Pages {
    uint32_t id[2];
  };
  auto pages_of = [&](uint32_t t) {
    Pages p;
#pragma unroll
    for (int b = 0; b < 2; ++b) p.id[b] = (uint32_t)table[min(t + 16 * b, end - 1) >> c.page_shift];
    return p;
  };
  // a lane's places in a block of 16 tokens: dims that a head does not have are read as its first ones, against zeros of q, and dropped
  constexpr uint32_t kSize = INT8 ? 1 : 2;
  uint32_t key_at[INT8 ? T::kSteps / 2 : T::kSteps];
#pragma unroll
  for (int s = 0; s < (INT8 ? T::kSteps / 2 : T::kSteps); ++s) {
    const uint32_t d0 = INT8 ? 64 * s + 16 * g : 32 * s + 8 * g;
    key_at[s] = kSize * (d0 < D ? d0 : 0);
  }
  const uint32_t val_at = kSize * (n * T::kVals < D ? n * T::kVals : 0);
  auto fetch = [&](T& x, uint32_t t, const Pages& p) {
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const uint32_t at = t + 16 * b;
      x.limit[b] = p.id[b] < c.n_pages && at < end ? min(end - at, 16u) : 0u;
      const uint32_t page = p.id[b] < c.n_pages ? p.id[b] : 0, slot = at & ((1u << c.page_shift) - 1);
      const uint64_t block = kSize * ((uint64_t)page * c.page_stride + kv * c.head_stride + slot * c.slot_stride);
      const char* key = c.k + block + kSize * (n * c.slot_stride);
#pragma unroll
      for (int s = 0; s < (INT8 ? T::kSteps / 2 : T::kSteps); ++s) load_words<4>(&x.k[b][4 * s], key + key_at[s]);
#pragma unroll
      for (int j = 0; j < 4; ++j) load_words<T::kValWords>(x.v[4 * b + j], c.v + block + (kSize * ((4 * g + j) * c.slot_stride) + val_at));
      if constexpr (INT8) {
        const uint64_t mark = (((uint64_t)page * c.kv_heads + kv) << c.page_shift) + slot + 4 * g;
        x.ks[b] = *(const float4*)(c.k_scale + mark);
        x.vs[b] = *(const float4*)(c.v_scale + mark);
      }
    }
  };
  auto take = [&](T& x, uint32_t t) {
    float p[8];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      f32x4 l = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < T::kSteps; ++s) {
        bf16x8 key;
        if constexpr (INT8) key = i8x8_to_bf16x8(make_uint2(x.k[b][2 * s], x.k[b][2 * s + 1]));
        else key = __builtin_bit_cast(bf16x8, make_uint4(x.k[b][4 * s], x.k[b][4 * s + 1], x.k[b][4 * s + 2], x.k[b][4 * s + 3]));
        l = __builtin_amdgcn_mfma_f32_16x16x32_bf16(key, q[s][0], l, 0, 0, 0);
        l = __builtin_amdgcn_mfma_f32_16x16x32_bf16(key, q[s][1], l, 0, 0, 0);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float v = ror8_sum(l[j]);
        if constexpr (INT8) v *= (&x.ks[b].x)[j];
        p[4 * b + j] = v;
      }
    }
    if (x.limit[0] < 16 || x.limit[1] < 16) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (4 * g + i % 4 >= x.limit[i / 4]) {
          p[i] = -INFINITY;
          if constexpr (INT8) (&x.vs[i / 4].x)[i % 4] = 0.f;
#pragma unroll
          for (int w = 0; w < T::kValWords; ++w) x.v[i][w] = 0;
        }
    }
    if constexpr (TRACK) {
      if (part == 0 && head < n_heads) {
        float* to = a.logits + ((uint64_t)r * a.heads + first_head + head) * c.capacity + t + 4 * g;
        *(float4*)to = make_float4(p[0], p[1], p[2], p[3]);
        if (t + 16 < end) *(float4*)(to + 16) = make_float4(p[4], p[5], p[6], p[7]);
      }
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
    bf16x8 pb;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float w = __builtin_amdgcn_exp2f(p[i] - base);
      total += w;
      if constexpr (INT8) w *= (&x.vs[i / 4].x)[i % 4];
      const __bf16 hi = (__bf16)w;
      pb[i] = part ? (__bf16)(w - (float)hi) : hi;
    }
#pragma unroll
    for (int b = 0; b < T::kVals; ++b) {
      uint32_t vt[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (INT8) {
          const float lo = (float)(int8_t)(x.v[2 * i][b / 4] >> (8 * (b % 4))), hi = (float)(int8_t)(x.v[2 * i + 1][b / 4] >> (8 * (b % 4)));
          vt[i] = __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
        } else {
          vt[i] = __builtin_amdgcn_perm(x.v[2 * i + 1][b / 2], x.v[2 * i][b / 2], b % 2 ? 0x07060302u : 0x05040100u);
        }
      }
      o[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, make_uint4(vt[0], vt[1], vt[2], vt[3])), pb, o[b], 0, 0, 0);
    }
  };
  const uint32_t first = begin + wave * kTile;
  if (first < end) {
    const uint32_t last = first + (end - 1 - first) / kUnit * kUnit;
    T x, y;
    fetch(x, first, pages_of(first));
    Pages next = pages_of(min(first + kUnit, last));
    for (uint32_t t = first;; t += 2 * kUnit) {
      fetch(y, min(t + kUnit, last), next);
      next = pages_of(min(t + 2 * kUnit, last));
      take(x, t);
      if (t == last) break;
      fetch(x, min(t + 2 * kUnit, last), next);
      next = pages_of(min(t + 3 * kUnit, last));
      take(y, t + kUnit);
      if (t + kUnit == last) break;
    }
  }

  // join the wavefronts: lane (g, head) holds dims (4 g + j) * kVals + b of the head, halves of p beside each other
  total += __shfl_xor(total, 16);
  total += __shfl_xor(total, 32);
  if (lane < kHeads) lds_max[wave * kHeads + lane] = top, lds_total[wave * kHeads + lane] = total;
#pragma unroll
  for (int b = 0; b < T::kVals; b += 4)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float4 v = make_float4(ror8_sum(o[b][j]), ror8_sum(o[b + 1][j]), ror8_sum(o[b + 2][j]), ror8_sum(o[b + 3][j]));
      if (part == 0) *(float4*)&lds_sum[(wave * kHeads + head) * (DIM + 4) + (4 * g + j) * T::kVals + b] = v;
    }
  __syncthreads();
  // the workgroups among which this (row, chunk) is cut
  const uint32_t pair_first = row_first + pair * units, group0 = pair_first / share, parts = (pair_first + units - 1) / share - group0 + 1;
  const uint64_t slot_floats = kHeads * (D + 2);
  auto slot_of = [&](uint32_t group) { return a.partials + (2 * (uint64_t)group + (group * share >= pair_first ? 0 : 1)) * slot_floats; };
  auto finish = [&](uint32_t h, uint32_t d, float sum, float m, float sum_p) {
    const float inv = sum_p == 0.f ? 0.f : 1.f / sum_p;
    a.out[r * a.out_stride + (first_head + h) * D + d] = (uint16_t)pack_bf16(sum * inv, 0.f);
    if (TRACK && d == 0) a.stats[(uint64_t)r * a.heads + first_head + h] = make_float2(m == -INFINITY ? 0.f : m, inv);
  };
  // one of n parts' sums, maxima and totals in LDS, [part][head][DIM + 4] from head h0 on -> the whole
  auto joined = [&](uint32_t parts_n, uint32_t h_n, uint32_t h0, uint32_t i, auto&& put) {
    const uint32_t h = i / D, d = i % D;
    float m = -INFINITY, sum = 0.f, sum_p = 0.f;
    for (uint32_t w = 0; w < parts_n; ++w) m = fmaxf(m, lds_max[w * kHeads + h0 + h]);
    const float base = m == -INFINITY ? 0.f : m;
    for (uint32_t w = 0; w < parts_n; ++w) {
      const float f = __builtin_amdgcn_exp2f(lds_max[w * kHeads + h0 + h] - base);
      sum = fmaf(f, lds_sum[(w * h_n + h) * (DIM + 4) + d], sum);
      sum_p = fmaf(f, lds_total[w * kHeads + h0 + h], sum_p);
    }
    put(h0 + h, d, sum, m, sum_p);
  };
  if (parts == 1) {
    for (uint32_t i = threadIdx.x; i < n_heads * D; i += kAttendThreads) joined(kAttendWaves, kHeads, 0, i, finish);
  } else {
    typedef __attribute__((address_space(1))) float global_f32;
    typedef __attribute__((address_space(1))) uint32_t global_u32;
    float* mine = slot_of(blockIdx.x);
    auto leave = [&](float* p, float v) { __hip_atomic_store((global_f32*)p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
    for (uint32_t i = threadIdx.x; i < n_heads * D; i += kAttendThreads)
      joined(kAttendWaves, kHeads, 0, i, [&](uint32_t h, uint32_t d, float sum, float m, float sum_p) {
        leave(mine + h * D + d, sum);
        if (d == 0) leave(mine + kHeads * D + 2 * h, m), leave(mine + kHeads * D + 2 * h + 1, sum_p);
      });
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // the stores have reached the level that the device shares
    __syncthreads();
    global_u32* arrived = (global_u32*)(a.arrived + (uint64_t)r * a.chunks + pair);
    if (threadIdx.x == 0) lds_before = __hip_atomic_fetch_add(arrived, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    if (lds_before == parts - 1) {   // the others' parts are in
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
      if (threadIdx.x == 0) __hip_atomic_store(arrived, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      // groups of DIM / 4 lanes take every kGroups-th part, four dims a lane, all heads
      constexpr uint32_t kLanes = DIM / 4, kGroups = kAttendThreads / kLanes, kBatch = kAttendWaves * kHeads / kGroups;
      const uint32_t mine_of = threadIdx.x / kLanes, d0 = threadIdx.x % kLanes * 4;
      float4 sum[kHeads];
      float m[kHeads], sum_p[kHeads];
#pragma unroll
      for (int h = 0; h < kHeads; ++h) sum[h] = make_float4(0.f, 0.f, 0.f, 0.f), m[h] = -INFINITY, sum_p[h] = 0.f;
      for (uint32_t v = mine_of; v < parts; v += kGroups) {
        const float* from = slot_of(group0 + v);
#pragma unroll
        for (uint32_t h = 0; h < kHeads; ++h)
          if (h < n_heads) {
            const float4 s = d0 < D ? *(const float4*)(from + h * D + d0) : make_float4(0.f, 0.f, 0.f, 0.f);
            const float2 st = *(const float2*)(from + kHeads * D + 2 * h);
            const float to = fmaxf(m[h], st.x), base = to == -INFINITY ? 0.f : to;
            const float f = __builtin_amdgcn_exp2f(m[h] - base), e = __builtin_amdgcn_exp2f(st.x - base);
            m[h] = to;
            sum_p[h] = sum_p[h] * f + st.y * e;
            sum[h].x = sum[h].x * f + s.x * e, sum[h].y = sum[h].y * f + s.y * e;
            sum[h].z = sum[h].z * f + s.z * e, sum[h].w = sum[h].w * f + s.w * e;
          }
      }
      if (threadIdx.x % kLanes == 0)
#pragma unroll
        for (int h = 0; h < kHeads; ++h) lds_max[mine_of * kHeads + h] = m[h], lds_total[mine_of * kHeads + h] = sum_p[h];
      for (uint32_t h0 = 0; h0 < n_heads; h0 += kBatch) {
        __syncthreads();
#pragma unroll
        for (int h = 0; h < kHeads; ++h)
          if (h >= (int)h0 && h < (int)(h0 + kBatch)) *(float4*)&lds_sum[(mine_of * kBatch + h - h0) * (DIM + 4) + d0] = sum[h];
        __syncthreads();
        const uint32_t some = min(kBatch, n_heads - h0);
        for (uint32_t i = threadIdx.x; i < some * D; i += kAttendThreads) joined(kGroups, kBatch, h0, i, finish);
      }
    }
  }
  __syncthreads();   // LDS is free again
  pos += unit_end - unit;
  if (pos == row_first + units * a.chunks) row_first = pos, ++r;
  }
}

// Adds the weights of all rows of a sequence to its slots' scores, rows and heads in order.
__global__ __launch_bounds__(256) void k_attend_scores(CacheView c, AttendView a) {
  const uint32_t slot = blockIdx.x * 256 + threadIdx.x, kv = blockIdx.y, s = blockIdx.z;
  if (slot >= c.capacity) return;
  const uint64_t at = ((uint64_t)s * c.kv_heads + kv) * c.capacity + slot;
  float sum = 0.f;
  bool any = false;
  const uint32_t r0 = a.seqs ? 0 : s, r1 = a.seqs ? a.rows : min(a.rows, s + 1);
  for (uint32_t r = r0; r < r1; ++r) {
    if (a.seqs && a.seqs[r] != (int32_t)s) continue;
    if ((int64_t)slot >= (int64_t)a.lengths[r]) continue;
    any = true;
    for (uint32_t h = kv * a.group; h < (kv + 1) * a.group; ++h) {
      const float2 st = a.stats[(uint64_t)r * a.heads + h];
      sum += __builtin_amdgcn_exp2f(a.logits[((uint64_t)r * a.heads + h) * c.capacity + slot] - st.x) * st.y;
    }
  }
  if (any) c.scores[at] += sum;
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
  if (a->accumulate && !c->scores) return refuse(TQ_E_INVALID_ARG, who + ": the cache has no scores to add to");
  if (!(a->scale > 0.f) || !(a->scale < INFINITY)) return refuse(TQ_E_INVALID_ARG, who + ": scale must be positive");
  const uint32_t group = a->heads / c->kv_heads;
  l->chunks = c->kv_heads * ((group + kHeads - 1) / kHeads);
  const uint64_t most = (uint64_t)a->rows * l->chunks * ((c->capacity + kUnit - 1) / kUnit);   // units, if all rows are full
  if (most >= (1u << 31) - kMaxGroups) return refuse(TQ_E_UNSUPPORTED, who + ": rows * heads * capacity is beyond what one call takes");
  l->groups = (uint32_t)std::min<uint64_t>(kMaxGroups, std::max<uint64_t>(1, (most + kMinShare - 1) / kMinShare));
  auto place = [&](uint64_t n) {
    const uint64_t at = l->bytes;
    l->bytes += (n + 255) / 256 * 256;
    return at;
  };
  l->bytes = 0;
  l->arrived = place((uint64_t)a->rows * l->chunks * 4);
  l->partials = place((uint64_t)l->groups * 2 * kHeads * (c->head_dim + 2) * 4);
  l->logits = a->accumulate ? place((uint64_t)a->rows * a->heads * c->capacity * 4) : 0;
  l->stats = a->accumulate ? place((uint64_t)a->rows * a->heads * 8) : 0;
  return TQ_OK;
}

template <int DIM>
void launch_attend(const CacheView& c, const AttendView& a, uint32_t groups, bool int8, bool track, hipStream_t stream) {
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(groups), dim3(kAttendThreads), 0, stream, c, a); };
  if (int8) track ? go(k_attend<DIM, true, true>) : go(k_attend<DIM, true, false>);
  else track ? go(k_attend<DIM, false, true>) : go(k_attend<DIM, false, false>);
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
                     a->scale * kLog2e, a->rows, a->heads, a->heads / c.kv_heads, l.chunks, q16};
  const bool int8 = cache->type == TQ_INT8;
  hipStream_t s = (hipStream_t)stream;
  if (c.head_dim <= 64) launch_attend<64>(c, v, l.groups, int8, a->accumulate, s);
  else if (c.head_dim <= 128) launch_attend<128>(c, v, l.groups, int8, a->accumulate, s);
  else launch_attend<256>(c, v, l.groups, int8, a->accumulate, s);
  if (a->accumulate) hipLaunchKernelGGL(k_attend_scores, dim3((c.capacity + 255) / 256, c.kv_heads, c.n_seqs), dim3(256), 0, s, c, v);
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
