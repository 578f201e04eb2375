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

constexpr int kAttendWaves = 4, kTile = 32, kHeads = 8;   // kHeads: query heads of a workgroup
constexpr uint32_t kSplitTokens = 1024;
constexpr float kLog2e = 1.4426950408889634f;

struct AttendView {
  const void* q;
  uint16_t* out;
  const int32_t *seqs, *lengths;
  float* partials;   // [row][chunk][split]: kHeads x (head_dim sums, maximum, total)
  float* logits;     // [row][head][capacity], in units of log 2 (accumulate)
  float2* stats;     // [row][head]: maximum and 1 / total of the whole row (accumulate)
  uint64_t q_stride, out_stride;
  float scale;       // times log2(e)
  uint32_t rows, heads, group, chunks, splits;   // chunks: workgroups per split that share its keys' head, times kv_heads
};

__device__ __forceinline__ float ror8_sum(float v) {   // v of this lane + v of the lane 8 columns on
  return v + __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), 0x128, 0xf, 0xf, true));
}

__device__ __forceinline__ uint32_t row_length(const CacheView& c, const AttendView& a, uint32_t r, uint32_t* seq) {
  const int32_t s = a.seqs ? a.seqs[r] : (int32_t)r;
  *seq = (uint32_t)s < c.n_seqs ? (uint32_t)s : 0;
  return (uint32_t)s < c.n_seqs ? (uint32_t)min(max(a.lengths[r], 0), (int32_t)c.capacity) : 0;
}

template <int DIM, bool INT8>
struct Tile {
  static constexpr int kSteps = DIM / 32, kVals = DIM / 16;   // contraction steps of the logits; a lane's dims of a value
  static constexpr int kKeyWords = INT8 ? kSteps * 2 : kSteps * 4, kValWords = INT8 ? kVals / 4 : kVals / 2;
  uint32_t k[2][kKeyWords], v[8][kValWords];
  float ks[8], vs[8];
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

// One (row, key/value head and chunk of its query heads, split of the tokens) -> maximum, total and weighted sum of values.
template <int DIM, bool INT8, bool Q16, bool TRACK>
__global__ __launch_bounds__(kAttendWaves * 64) void k_attend_split(CacheView c, AttendView a) {
  using T = Tile<DIM, INT8>;
  __shared__ float lds_sum[kAttendWaves][kHeads][DIM + 4], lds_max[kAttendWaves][kHeads], lds_total[kAttendWaves][kHeads];
  const uint32_t split = blockIdx.x, r = blockIdx.z, per_kv = a.chunks / c.kv_heads;
  const uint32_t kv = blockIdx.y / per_kv, chunk = blockIdx.y % per_kv;
  const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane / 16, n = lane % 16, head = n % 8, part = n / 8;
  uint32_t seq;
  const uint32_t length = row_length(c, a, r, &seq), begin = split * kSplitTokens, end = min(length, begin + kSplitTokens);
  if (begin >= end) return;
  const uint32_t D = c.head_dim;
  const uint32_t first_head = kv * a.group + chunk * kHeads, n_heads = min((uint32_t)kHeads, a.group - chunk * kHeads);
  const int32_t* table = c.tables + (uint64_t)seq * c.table_stride;

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
        x = (Q16 ? bf16_value(((const uint16_t*)a.q)[at]) : ((const float*)a.q)[at]) * a.scale;
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

  for (uint32_t t = begin + wave * kTile; t < end; t += kAttendWaves * kTile) {
    T x;
    uint32_t limit[2];   // tokens of a 16-token block that take part
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const uint32_t at = t + 16 * b;
      uint32_t page = at < end ? (uint32_t)table[at >> c.page_shift] : c.n_pages;
      limit[b] = page < c.n_pages ? min(end - at, 16u) : 0u;
      if (page >= c.n_pages) page = 0;
      const uint32_t slot = at & ((1u << c.page_shift) - 1);
      const uint64_t block = (uint64_t)page * c.page_stride + kv * c.head_stride + slot * c.slot_stride;
      const uint64_t size = INT8 ? 1 : 2;
      const char* key = c.k + size * (block + n * c.slot_stride);
#pragma unroll
      for (int s = 0; s < T::kSteps; s += INT8 ? 2 : 1) {
        const uint32_t d0 = INT8 ? 32 * s + 16 * g : 32 * s + 8 * g;
        uint32_t* to = &x.k[b][(INT8 ? s / 2 : s) * 4];
        if (d0 < D) load_words<4>(to, key + size * d0);
        else to[0] = to[1] = to[2] = to[3] = 0;
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t d0 = n * T::kVals;
        if (d0 < D) load_words<T::kValWords>(x.v[4 * b + j], c.v + size * (block + (4 * g + j) * c.slot_stride + d0));
        else
#pragma unroll
          for (int w = 0; w < T::kValWords; ++w) x.v[4 * b + j][w] = 0;
      }
      if constexpr (INT8) {
        const uint64_t mark = (((uint64_t)page * c.kv_heads + kv) << c.page_shift) + slot + 4 * g;
        const float4 ks = *(const float4*)(c.k_scale + mark), vs = *(const float4*)(c.v_scale + mark);
        x.ks[4 * b] = ks.x, x.ks[4 * b + 1] = ks.y, x.ks[4 * b + 2] = ks.z, x.ks[4 * b + 3] = ks.w;
        x.vs[4 * b] = vs.x, x.vs[4 * b + 1] = vs.y, x.vs[4 * b + 2] = vs.z, x.vs[4 * b + 3] = vs.w;
      }
    }
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
        if constexpr (INT8) v *= x.ks[4 * b + j];
        p[4 * b + j] = v;
      }
    }
    if (limit[0] < 16 || limit[1] < 16) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (4 * g + i % 4 >= limit[i / 4]) {
          p[i] = -INFINITY;
          if constexpr (INT8) x.vs[i] = 0.f;
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
      if constexpr (INT8) w *= x.vs[i];
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
  }

  // join the wavefronts: lane (g, head) holds dims (4 g + j) * kVals + b of the head, halves of p beside each other
  total += __shfl_xor(total, 16);
  total += __shfl_xor(total, 32);
  if (lane < kHeads) lds_max[wave][lane] = top, lds_total[wave][lane] = total;
#pragma unroll
  for (int b = 0; b < T::kVals; ++b)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float v = ror8_sum(o[b][j]);
      if (part == 0) lds_sum[wave][head][(4 * g + j) * T::kVals + b] = v;
    }
  __syncthreads();
  float* to = a.partials + (((uint64_t)r * a.chunks + blockIdx.y) * a.splits + split) * kHeads * (D + 2);
  for (uint32_t i = threadIdx.x; i < n_heads * D; i += kAttendWaves * 64) {
    const uint32_t h = i / D, d = i % D;
    float m = -INFINITY, sum = 0.f, all = 0.f;
#pragma unroll
    for (int w = 0; w < kAttendWaves; ++w) m = fmaxf(m, lds_max[w][h]);
    const float base = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int w = 0; w < kAttendWaves; ++w) {
      const float f = __builtin_amdgcn_exp2f(lds_max[w][h] - base);
      sum = fmaf(f, lds_sum[w][h][d], sum);
      all = fmaf(f, lds_total[w][h], all);
    }
    to[h * D + d] = sum;
    if (d == 0) to[kHeads * D + 2 * h] = m, to[kHeads * D + 2 * h + 1] = all;
  }
}

// Joins a row's splits: one workgroup per query head.
__global__ __launch_bounds__(64) void k_attend_join(CacheView c, AttendView a) {
  const uint32_t h = blockIdx.x, r = blockIdx.y, D = c.head_dim;
  const uint32_t kv = h / a.group, per_kv = a.chunks / c.kv_heads, chunk = kv * per_kv + h % a.group / kHeads, in = h % a.group % kHeads;
  uint32_t seq;
  const uint32_t length = row_length(c, a, r, &seq), n = (length + kSplitTokens - 1) / kSplitTokens;
  const float* from = a.partials + ((uint64_t)r * a.chunks + chunk) * a.splits * kHeads * (D + 2);
  const uint64_t step = kHeads * (D + 2);
  float m = -INFINITY;
  for (uint32_t s = 0; s < n; ++s) m = fmaxf(m, from[s * step + kHeads * D + 2 * in]);
  const float base = m == -INFINITY ? 0.f : m;
  float all = 0.f;
  for (uint32_t s = 0; s < n; ++s) all = fmaf(__builtin_amdgcn_exp2f(from[s * step + kHeads * D + 2 * in] - base), from[s * step + kHeads * D + 2 * in + 1], all);
  const float inv = all == 0.f ? 0.f : 1.f / all;
  for (uint32_t d = threadIdx.x; d < D; d += 64) {
    float sum = 0.f;
    for (uint32_t s = 0; s < n; ++s) sum = fmaf(__builtin_amdgcn_exp2f(from[s * step + kHeads * D + 2 * in] - base), from[s * step + in * D + d], sum);
    a.out[r * a.out_stride + h * D + d] = (uint16_t)pack_bf16(sum * inv, 0.f);
  }
  if (a.stats && threadIdx.x == 0) a.stats[(uint64_t)r * a.heads + h] = make_float2(base, inv);
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
  uint64_t partials, logits, stats, bytes;   // offsets
  uint32_t chunks, splits;
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
  l->splits = (c->capacity + kSplitTokens - 1) / kSplitTokens;
  auto place = [&](uint64_t n) {
    const uint64_t at = l->bytes;
    l->bytes += (n + 255) / 256 * 256;
    return at;
  };
  l->bytes = 0;
  l->partials = place((uint64_t)a->rows * l->chunks * l->splits * kHeads * (c->head_dim + 2) * 4);
  l->logits = a->accumulate ? place((uint64_t)a->rows * a->heads * c->capacity * 4) : 0;
  l->stats = a->accumulate ? place((uint64_t)a->rows * a->heads * 8) : 0;
  return TQ_OK;
}

template <int DIM>
void launch_split(const CacheView& c, const AttendView& a, bool int8, bool q16, bool track, hipStream_t stream) {
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(a.splits, a.chunks, a.rows), dim3(kAttendWaves * 64), 0, stream, c, a); };
  auto pick = [&](auto i8, auto q) {
    track ? go(k_attend_split<DIM, decltype(i8)::value, decltype(q)::value, true>) : go(k_attend_split<DIM, decltype(i8)::value, decltype(q)::value, false>);
  };
  if (int8) q16 ? pick(std::true_type(), std::true_type()) : pick(std::true_type(), std::false_type());
  else q16 ? pick(std::false_type(), std::true_type()) : pick(std::false_type(), std::false_type());
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
  const AttendView v{a->q, (uint16_t*)a->out, a->seqs, a->lengths, (float*)(ws + l.partials), (float*)(ws + l.logits),
                     a->accumulate ? (float2*)(ws + l.stats) : nullptr, a->q_stride ? a->q_stride : row, a->out_stride ? a->out_stride : row,
                     a->scale * kLog2e, a->rows, a->heads, a->heads / c.kv_heads, l.chunks, l.splits};
  const bool int8 = cache->type == TQ_INT8;
  hipStream_t s = (hipStream_t)stream;
  if (c.head_dim <= 64) launch_split<64>(c, v, int8, q16, a->accumulate, s);
  else if (c.head_dim <= 128) launch_split<128>(c, v, int8, q16, a->accumulate, s);
  else launch_split<256>(c, v, int8, q16, a->accumulate, s);
  hipLaunchKernelGGL(k_attend_join, dim3(a->heads, a->rows), dim3(64), 0, s, c, v);
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
