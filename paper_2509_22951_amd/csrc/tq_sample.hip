// One token per row, drawn from its logits (tq_sample).
#include <algorithm>

#include "tq_cache_view.h"

namespace tq {
namespace {

constexpr uint32_t kMostVocab = 1u << 20, kThreads = 256, kFew = 2, kMany = 4;   // kFew, kMany: four logits each, of a thread
constexpr uint32_t kApart = 32;   // words from one counter to the next, in a cache line of its own
constexpr uint32_t kMostParts = kMostVocab / (4 * kFew * kThreads);
constexpr uint32_t kBinThreads = 1024, kBins = 2048, kBinsPerUnit = 32, kListed = 2048;   // bins of (largest - logit) / temperature; keys held in LDS

// What the launches leave each other, for every row.
struct Notes {
  uint64_t* keys;      // [row][part]: the first token's key
  uint64_t* mass;      // [row][kBins]: weights of a bin
  uint32_t* count;     // [row][kBins]: tokens of a bin
  double* kept;        // [row][part]: weight of what is kept beyond doubt; of an open row, of all tokens relative to the part's first one
  uint32_t* listed;    // [row][part]: tokens in the part's list
  uint64_t* list;      // [row][vocab]: of every part, where its tokens begin, the keys of those in the bin that the cut lies in
  uint32_t* done;      // [row * kApart]: workgroups that are
};

struct SampleView {
  const float* logits;
  const float *temperature, *top_p, *min_p, *uniform;
  const int32_t* top_k;
  int32_t* tokens;
  float* probs;
  Notes notes;
  uint64_t stride;
  uint32_t rows, vocab, parts, mass_bits;   // weights are summed in units of 2^-mass_bits where the order of summation is not fixed
};

// Keys that compare as the tokens' order does: by logit (NaN lowest, -0 as 0), equal ones by number, the lowest first.
__device__ __forceinline__ uint32_t rank_of(float l) {
  if (l != l) return 0;
  const uint32_t b = __float_as_uint(l + 0.f);
  return b >> 31 ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ uint64_t key_of(float l, uint32_t i) { return (uint64_t)rank_of(l) << 32 | (uint32_t)~i; }

__device__ __forceinline__ float logit_of_rank(uint32_t rank) { return __uint_as_float(rank >> 31 ? rank & 0x7FFFFFFFu : ~rank); }

// exp((l - top) / temperature) as 2^y, y = (l - top) * (log2(e) / temperature): 2^n times the series of 2^f, ln(2)^k / k! f^k, for |f| <= 1/2, whose 13 terms leave 2^-52 of it.  Few
// instructions and no branches: a workgroup runs through them once, and what does not fit the instruction cache is waited for.  (Its coefficients are in scalar registers; as literals
// each costs two moves, and 64 rows of 128256 without filters took 131 us.)
struct Weigher {
  double top, per_unit, c[13];
  float top32;
  __device__ __forceinline__ Weigher(float t, float temperature)
      : top(t), per_unit(1.4426950408889634074 / (double)temperature),
        c{1., 6.9314718055994531e-01, 2.4022650695910071e-01, 5.5504108664821580e-02, 9.6181291076284772e-03, 1.3333558146428443e-03, 1.5403530393381609e-04, 1.5252733804059840e-05,
          1.3215486790144309e-06, 1.0178086009239699e-07, 7.0549116208011233e-09, 4.4455382718708115e-10, 2.5678435993488205e-11},
        top32(t) {
#pragma unroll
    for (int k = 0; k < 13; ++k) asm("" : "+s"(c[k]));
  }
  __device__ __forceinline__ double operator()(float l) const {
    const double y = fmax(((double)l - top) * per_unit, -1100.), n = rint(y), f = y - n;
    double s = c[12];
#pragma unroll
    for (int k = 11; k >= 0; --k) s = fma(s, f, c[k]);
    s = ldexp(s, (int)n);
    s = l == top32 ? 1. : s;
    return l > -INFINITY ? s : 0.;
  }
  // Whether that is more than zero, without the series (to less than half of the smallest number of 64 bits: zero).
  __device__ __forceinline__ bool any(float l) const { return l == top32 || ((double)l - top) * per_unit > -1075.; }
};

// How a row is to be drawn from.
struct Filter {
  float top, temperature, per_bin, p, least;   // per_bin: bins of a unit of the logit
  uint32_t first, k;
  bool drawn, by_rank, by_mass;   // drawn: not merely the first token; by_rank, by_mass: top_k or top_p leaves something out
};

// A value of 4 or 8 bytes from another lane of the same wavefront (0 where there is none), within the vector registers.  (Shuffles through LDS: 14.2 us for one row's last launch, 23.7 for 16
// rows', in place of 11.9 and 20.8.)
template <int CONTROL, int ROWS, bool ZERO, typename T>
__device__ __forceinline__ T from_lane(T v) {
  if constexpr (sizeof(T) == 4) {
    return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CONTROL, ROWS, 0xf, ZERO));
  } else {
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CONTROL, ROWS, 0xf, ZERO), hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(u >> 32), CONTROL, ROWS, 0xf, ZERO);
    return __builtin_bit_cast(T, (uint64_t)hi << 32 | lo);
  }
}
template <typename T>
__device__ __forceinline__ T of_lane(T v, uint32_t lane) {   // (the same for all lanes)
  if constexpr (sizeof(T) == 4) {
    return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
  } else {
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    return __builtin_bit_cast(T, (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(u >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)u, lane));
  }
}
// Of a wavefront's lanes up to and with each, joined in the same order every time; 0 joined with a value is that value.  By all lanes.
template <typename T, typename JOIN>
__device__ __forceinline__ T wave_joined(T v, JOIN join) {
  v = join(v, from_lane<0x111, 0xf, true>(v));
  v = join(v, from_lane<0x112, 0xf, true>(v));
  v = join(v, from_lane<0x114, 0xf, true>(v));
  v = join(v, from_lane<0x118, 0xf, true>(v));
  v = join(v, from_lane<0x142, 0xa, false>(v));   // lane 15 of a row to the next one
  return join(v, from_lane<0x143, 0xc, false>(v));   // lane 31 to the upper half
}
template <typename T>
__device__ __forceinline__ T wave_upto(T v) { return wave_joined(v, [](T x, T y) { return x + y; }); }
template <typename T>
__device__ __forceinline__ T wave_sum(T v) { return of_lane(wave_upto(v), 63); }
template <typename T>
__device__ __forceinline__ T wave_most(T v) { return of_lane(wave_joined(v, [](T x, T y) { return max(x, y); }), 63); }
__device__ __forceinline__ uint32_t wave_least(uint32_t v) { return ~wave_most(~v); }

// What the caller asks of a row.  (Four loads at once, where conditions would put them behind each other.)
struct Asked {
  float temperature, p, least;
  int32_t k;
};
__device__ __forceinline__ Asked asked_of(const SampleView& a, uint32_t r) {
  const float t = (a.temperature ? a.temperature : a.uniform)[r], p = (a.top_p ? a.top_p : a.uniform)[r], least = (a.min_p ? a.min_p : a.uniform)[r];
  const int32_t k = (a.top_k ? a.top_k : (const int32_t*)a.uniform)[r];
  return Asked{a.temperature ? t : 1.f, a.top_p ? p : 1.f, a.min_p ? least : 0.f, a.top_k ? k : 0};
}
__device__ __forceinline__ bool limited(const Asked& x, uint32_t vocab) { return x.k > 0 && (uint32_t)x.k < vocab; }
// A row that is drawn from without filters: its parts' weights are summed in the first launch already, relative to their own first tokens'.
__device__ __forceinline__ bool is_open(const Asked& x, uint32_t vocab) { return x.temperature > 0.f && !limited(x, vocab) && !(x.p < 1.f) && !(x.least > 0.f); }

// From the first token's key.
__device__ __forceinline__ Filter filter_from(const Asked& x, uint32_t vocab, uint64_t best) {
  Filter f;
  f.temperature = x.temperature;
  f.per_bin = (float)kBinsPerUnit / f.temperature;
  f.p = x.p, f.least = x.least;
  f.first = ~(uint32_t)best;
  f.top = best >> 32 ? logit_of_rank((uint32_t)(best >> 32)) : -INFINITY;
  f.k = limited(x, vocab) ? (uint32_t)x.k : vocab;
  f.drawn = f.top > -INFINITY && f.temperature > 0.f;
  f.by_rank = f.k < vocab, f.by_mass = f.p < 1.f;
  return f;
}
// The largest of all threads' keys (by all threads; slots: one per wavefront).
__device__ __forceinline__ uint64_t largest_of(uint64_t best, uint64_t* slots) {
  best = wave_most(best);
  if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = best;
  __syncthreads();
  best = slots[0];
  for (uint32_t w = 1; w < blockDim.x / 64; ++w) best = max(best, slots[w]);
  return best;
}
__device__ __forceinline__ Filter filter_of(const SampleView& a, uint32_t r, const Asked& x, uint64_t* slots) {
  uint64_t best = 0;
  for (uint32_t i = threadIdx.x; i < a.parts; i += blockDim.x) best = max(best, a.notes.keys[(uint64_t)r * a.parts + i]);
  return filter_from(x, a.vocab, largest_of(best, slots));
}

// Four neighbouring logits; those beyond the row are masked.
__device__ __forceinline__ void four_of(const float* row, uint32_t i, uint32_t n, float (&v)[4]) {
  if (i + 4 <= n) {
    const f32x4_any d = *(const f32x4_any*)(row + i);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = d[j];
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = i + j < n ? row[i + j] : __builtin_nanf("");
  }
}

// The bin of a logit: never lower for a smaller one, since each step rounds in order.
__device__ __forceinline__ float distance_of(const Filter& f, float l) {
  const float d = (f.top - l) * f.per_bin;
  return l == f.top ? 0.f : l > -INFINITY ? d : INFINITY;
}
__device__ __forceinline__ uint32_t bin_of(float distance) { return distance < (float)(kBins - 1) ? (uint32_t)distance : kBins - 1; }

// Every part is 1024 * CHUNKS tokens: of few rows small ones, so that there is a workgroup for every compute unit; of many rows larger ones.
template <int CHUNKS>
constexpr uint32_t kPart = 4 * CHUNKS * kThreads;

// First launch: the first token of every part, and an open row's weights; bins and counters are cleared for the next ones.
//
// Bound: a launch and a wait for few rows (3.1 us, at the least 2.0); for many the reading, and of open rows the weights, which a part's largest logit has to be known for: 64 rows of 128256 7.9 us (7.6),
// 16.4 (14.6) if open.
template <int CHUNKS>
__global__ __launch_bounds__(kThreads) void k_sample_first(SampleView a) {
  __shared__ uint64_t slots[kThreads / 64];
  __shared__ double sums[kThreads / 64];
  const uint32_t part = blockIdx.x, r = blockIdx.y, tid = threadIdx.x;
  const float* row = a.logits + r * a.stride;
  const Asked asked = asked_of(a, r);
  float v[CHUNKS][4];
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) four_of(row, part * kPart<CHUNKS> + 4 * (c * kThreads + tid), a.vocab, v[c]);
  for (uint32_t i = part * kThreads + tid; i < kBins; i += a.parts * kThreads) a.notes.mass[(uint64_t)r * kBins + i] = 0, a.notes.count[(uint64_t)r * kBins + i] = 0;
  if (part == 0 && tid == 0) a.notes.done[(uint64_t)r * kApart] = 0;
  uint64_t best = 0;
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t i = part * kPart<CHUNKS> + 4 * (c * kThreads + tid) + j;
      if (i < a.vocab) best = max(best, key_of(v[c][j], i));
    }
  best = largest_of(best, slots);
  if (tid == 0) a.notes.keys[(uint64_t)r * a.parts + part] = best;
  if (!is_open(asked, a.vocab)) return;
  const Weigher weight(logit_of_rank((uint32_t)(best >> 32)), asked.temperature);
  double sum = 0.;
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
    for (int j = 0; j < 4; ++j) sum += weight(v[c][j]);   // (NaN beyond the row)
  sum = wave_sum(sum);
  if ((tid & 63) == 0) sums[tid >> 6] = sum;
  __syncthreads();
  if (tid == 0) {
    for (uint32_t w = 1; w < kThreads / 64; ++w) sum += sums[w];
    a.notes.kept[(uint64_t)r * a.parts + part] = sum;
  }
}

// Second launch, for rows with top_k or top_p: tokens and weights of every bin.  PER tokens a thread.  Tokens without any weight, the masked ones, are left out: none of them is drawn
// whether it is kept or not, and a cut among all that a grammar leaves of a vocabulary, one row of 128256 logits with ten that are not masked and top_k 50, took 3800 us to find, now 17.
// Counts and weights are added up in LDS first, whole numbers both.  Bound: the parts' first keys -> weights -> additions in LDS -> additions in memory, behind each other: one row of 32000 logits 5.0 us (least: 4.5) with two
// tokens a thread, 6.7 with eight, which is what the many rows take that fill the card anyway (16 of 128256 8.0, 7.6).
template <int PER>
__global__ __launch_bounds__(kBinThreads) void k_sample_bins(SampleView a) {
  __shared__ uint64_t slots[kBinThreads / 64], lds_mass[kBins];
  __shared__ uint32_t lds_count[kBins];
  const uint32_t r = blockIdx.y, tid = threadIdx.x;
  const float* row = a.logits + r * a.stride;
  // (before anything is asked for: of a row without these filters, and of a greedy one, nothing is read)
  const Asked asked = asked_of(a, r);
  if (!(limited(asked, a.vocab) || asked.p < 1.f) || !(asked.temperature > 0.f)) return;
  const uint32_t first = blockIdx.x * (PER * kBinThreads);
  float v[PER];
  auto token = [&](int j) { return PER == 8 ? first + j / 4 * (4 * kBinThreads) + 4 * tid + j % 4 : first + j * kBinThreads + tid; };
  if constexpr (PER == 8) {
    four_of(row, token(0), a.vocab, *(float(*)[4])&v[0]), four_of(row, token(4), a.vocab, *(float(*)[4])&v[4]);
  } else {
#pragma unroll
    for (int j = 0; j < PER; ++j) v[j] = token(j) < a.vocab ? row[token(j)] : 0.f;
  }
  for (uint32_t b = tid; b < kBins; b += kBinThreads) lds_mass[b] = 0, lds_count[b] = 0;
  const Filter f = filter_of(a, r, asked, slots);
  if (!f.drawn || (!f.by_rank && !f.by_mass)) return;
  const Weigher weight(f.top, f.temperature);
  const double unit = (double)(1ull << a.mass_bits);
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const uint32_t b = bin_of(distance_of(f, v[j]));
    const uint64_t mass = (uint64_t)(weight(v[j]) * unit + 0.5);
    if (token(j) >= a.vocab || !weight.any(v[j])) continue;
    atomicAdd(&lds_count[b], 1u);
    if (f.by_mass) atomicAdd((unsigned long long*)&lds_mass[b], (unsigned long long)mass);
  }
  __syncthreads();
  for (uint32_t b = tid; b < kBins; b += kBinThreads)
    if (lds_count[b]) {
      atomicAdd(&a.notes.count[(uint64_t)r * kBins + b], lds_count[b]);
      if (f.by_mass) atomicAdd((unsigned long long*)&a.notes.mass[(uint64_t)r * kBins + b], (unsigned long long)lds_mass[b]);
    }
}

// The place in an order of bins, tokens and weights of a thread's neighbouring ones given, in which the last token lies that is kept: the first bin where a cut comes (bin kBins, if
// there are fewer tokens than that).  -> through LDS, by all threads.
struct Cut {
  uint32_t bin, above;      // tokens and weight ahead of the bin
  uint64_t above_mass;
};
template <int PER>
__device__ __forceinline__ Cut find_cut(const uint32_t (&count)[PER], const uint64_t (&mass)[PER], uint32_t above, uint64_t above_mass, uint32_t k, bool by_mass, double target,
                                        uint32_t* lds_n, uint64_t* lds_m, Cut* lds_cut) {
  const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  uint32_t n = 0;
  uint64_t m = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) n += count[i], m += mass[i];
  const uint32_t n_upto = wave_upto(n);
  const uint64_t m_upto = wave_upto(m);
  if (tid == 0) *lds_cut = Cut{kBins, 0, 0};
  __syncthreads();
  if (lane == 63) lds_n[wave] = n_upto, lds_m[wave] = m_upto;
  __syncthreads();
  uint32_t before = above + n_upto - n;
  uint64_t mass_before = above_mass + m_upto - m;
  for (uint32_t w = 0; w < wave; ++w) before += lds_n[w], mass_before += lds_m[w];
  // a bin's first token is kept if too few are ahead of it, and too little weight; the last such bin is the one that has the cut: where the next one with tokens is not
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const bool begins = before == 0 || (before < k && (!by_mass || (double)mass_before < target));
    const uint32_t after = before + count[i];
    const uint64_t mass_after = mass_before + mass[i];
    const bool goes_on = after < k && (!by_mass || (double)mass_after < target);
    if (count[i] && begins && !goes_on) *lds_cut = Cut{tid * PER + i, before, mass_before};
    before = after, mass_before = mass_after;
  }
  __syncthreads();
  return *lds_cut;
}

// Third launch: the weight of what is kept in every part, and the tokens of the bin that the cut lies in; the last workgroup of a row finds the cut and draws.  Of an open row, whose parts
// are summed, the first one draws.  A whole row (WHOLE: no more than a part) needs no launch ahead: its first token, its bins and its list are the workgroup's own.
//
// Bound: a chain of waits.  One row: logits, bins and the parts' first keys 1.8 us -> the bin of the cut 1.3 -> weights, sums over the workgroup, the list's stores 2.3 -> count 0.5 -> the parts' sums and lists 2 ->
// the cut within the bin 1 -> the part that has the token 0.9 -> its logits, weights once more 1.6: 11.7 us (least: 11.0) for 32000 tokens, beside 3.1 (2.0) and 5.0 (4.5) of the launches ahead.  16 rows of 128256 with filters:
// 20.2 us (19.8), beside 4.8 (4.2) and 8.0 (7.6) (read: 8 MB, 1.3 us).  64 open rows: 7.2 us (6.7), beside 16.4 (14.6) of the first launch (33 MB read, 5.2 us; weights, some 30 instructions of 64 bits
// each, 10) and 4.5 (3.8).  Why three
// launches: a row's largest logit is needed ahead of every weight that is compared with others, and the cut ahead of every sum; one workgroup per row, that needs no launch between, took 284 us for the first and 621 for the second.
template <int CHUNKS, bool WHOLE>
__global__ __launch_bounds__(kThreads) void k_sample_draw(SampleView a) {
  __shared__ uint64_t slots[kThreads / 64], lds_m[kThreads / 64], lds_keys[kListed], lds_mass[256], lds_more[kMostParts];
  __shared__ uint32_t lds_n[kThreads / 64], lds_count[256], lds_upto[kMostParts], lds_base, lds_done, lds_token, lds_last;
  __shared__ double lds_sum[kThreads / 64], lds_share;
  __shared__ Cut lds_cut;
  __shared__ uint64_t lds_bin_mass[WHOLE ? kBins : 1];
  __shared__ uint32_t lds_bin_count[WHOLE ? kBins : 1];
  const uint32_t part = blockIdx.y, r = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const float* row = a.logits + r * a.stride;
  // (the bins are asked for ahead of the largest logit: two waits for memory in place of three.  Of few rows all of it is asked for before it is known whether the row is open, 1.2 us less for one
  // of 32000 logits; of many, whose reading takes longer than the wait, after that: 64 open rows of 128256 9.5 us in place of 24.)
  constexpr int kBinsPer = kBins / kThreads;
  float v[CHUNKS][4];
  double w[CHUNKS][4];
  // (of a whole row neighbouring tokens, so that one sum over the threads is enough in the end)
  auto token_of = [&](int c, int j) { return WHOLE ? 4 * CHUNKS * tid + 4 * c + j : part * kPart<CHUNKS> + 4 * (c * kThreads + tid) + j; };
  uint32_t count[kBinsPer];
  uint64_t mass[kBinsPer];
  auto ask = [&] {
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) four_of(row, part * kPart<CHUNKS> + 4 * (c * kThreads + tid), a.vocab, v[c]);
#pragma unroll
    for (int i = 0; i < kBinsPer; ++i) {
      count[i] = a.notes.count[(uint64_t)r * kBins + tid * kBinsPer + i];
      mass[i] = a.notes.mass[(uint64_t)r * kBins + tid * kBinsPer + i];
    }
  };
  if constexpr (CHUNKS == kFew && !WHOLE) ask();
  const Asked asked = asked_of(a, r);
  const bool open = !WHOLE && is_open(asked, a.vocab);
  if (open && part) return;
  Filter f;
  if constexpr (WHOLE) {
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) four_of(row, token_of(c, 0), a.vocab, v[c]);
#pragma unroll
    for (int i = 0; i < kBinsPer; ++i) lds_bin_count[i * kThreads + tid] = 0, lds_bin_mass[i * kThreads + tid] = 0;
    uint64_t best = 0;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t i = token_of(c, j);
        if (i < a.vocab) best = max(best, key_of(v[c][j], i));
      }
    f = filter_from(asked, a.vocab, largest_of(best, slots));
  } else {
    if (CHUNKS != kFew && !open) ask();
    f = filter_of(a, r, asked, slots);
  }
  if (!f.drawn) {
    if (part == 0 && tid == 0) {
      a.tokens[r] = f.top > -INFINITY ? (int32_t)f.first : -1;
      if (a.probs) a.probs[r] = f.top > -INFINITY ? 1.f : 0.f;
    }
    return;
  }
  const Weigher weight(f.top, f.temperature);
  const double unit = (double)(1ull << a.mass_bits), least = (double)f.least;
  auto mass_of = [&](float l) { return (uint64_t)(weight(l) * unit + 0.5); };
  if constexpr (WHOLE)
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
      for (int j = 0; j < 4; ++j) w[c][j] = weight(v[c][j]);
  bool cuts = f.by_rank || f.by_mass;
  Cut cut{kBins, 0, 0};
  double target = 0.;
  if (cuts) {
    if constexpr (WHOLE) {
#pragma unroll
      for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t b = bin_of(distance_of(f, v[c][j]));
          const uint64_t its = (uint64_t)(w[c][j] * unit + 0.5);
          if (token_of(c, j) >= a.vocab || !weight.any(v[c][j])) continue;
          atomicAdd(&lds_bin_count[b], 1u);
          if (f.by_mass) atomicAdd((unsigned long long*)&lds_bin_mass[b], (unsigned long long)its);
        }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kBinsPer; ++i) count[i] = lds_bin_count[tid * kBinsPer + i], mass[i] = lds_bin_mass[tid * kBinsPer + i];
    }
    uint64_t all = 0;
#pragma unroll
    for (int i = 0; i < kBinsPer; ++i) all += mass[i];
    all = wave_sum(all);
    if (lane == 0) lds_m[wave] = all;
    __syncthreads();
    all = 0;
    for (uint32_t w = 0; w < kThreads / 64; ++w) all += lds_m[w];
    target = (double)f.p * (double)all;
    cut = find_cut<kBinsPer>(count, mass, 0, 0, f.k, f.by_mass, target, lds_n, lds_m, &lds_cut);
    cuts = cut.bin != kBins;
  }
  auto if_kept = [&](double w, uint32_t i) { return ((i == f.first) | !(w < least)) ? w : 0.; };   // of a token that no cut leaves out
  auto kept_weight = [&](float l, uint32_t i) { return if_kept(weight(l), i); };

  // this part
  double kept = 0.;   // (of a whole row)
  uint32_t all_listed = 0;
  if (!open) {
    const uint32_t part_first = part * kPart<CHUNKS>;
    double sum = 0.;
    uint32_t in_bin = 0;   // a bit per token
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t i = token_of(c, j);
        const uint32_t b = i >= a.vocab || !weight.any(v[c][j]) ? kBins + 1 : cuts ? bin_of(distance_of(f, v[c][j])) : 0;
        if constexpr (WHOLE) w[c][j] = if_kept(w[c][j], i);
        else w[c][j] = kept_weight(v[c][j], i);
        sum += b < cut.bin ? w[c][j] : 0.;
        in_bin |= (b == cut.bin ? 1u : 0u) << (4 * c + j);
      }
    const uint32_t n = (uint32_t)__builtin_popcount(in_bin);
    sum = wave_sum(sum);
    const uint32_t n_upto = wave_upto(n);
    __syncthreads();
    if (lane == 63) lds_n[wave] = n_upto, lds_sum[wave] = sum;
    __syncthreads();
    uint32_t at = n_upto - n, all_n = 0;
    for (uint32_t w = 0; w < kThreads / 64; ++w) {
      if (w < wave) at += lds_n[w];
      all_n += lds_n[w];
    }
    if (WHOLE || tid == 0)
      for (uint32_t w = 0; w < kThreads / 64; ++w) kept += lds_sum[w];
    if (!WHOLE && tid == 0) {
      __hip_atomic_store((uint64_t*)&a.notes.kept[(uint64_t)r * a.parts + part], __builtin_bit_cast(uint64_t, kept), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      __hip_atomic_store(&a.notes.listed[(uint64_t)r * a.parts + part], all_n, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    if (all_n) {
#pragma unroll
      for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t i = token_of(c, j);
          if (in_bin >> (4 * c + j) & 1) {
            if (WHOLE && at < kListed) lds_keys[at] = key_of(v[c][j], i);
            else __hip_atomic_store(&a.notes.list[(uint64_t)r * a.vocab + part_first + at], key_of(v[c][j], i), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            ++at;
          }
        }
    }
    // the stores have reached the level that the device shares; the last workgroup goes on with all of the row
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if constexpr (WHOLE) {
      all_listed = all_n;
    } else {
      if (tid == 0) lds_done = __hip_atomic_fetch_add(&a.notes.done[(uint64_t)r * kApart], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      __syncthreads();
      if (lds_done != a.parts - 1) return;
    }
  }

  // The cut within the bin: narrowed by a 256th of the bin, then by 8 bits of the key at a time, until few enough are left to compare all with each other.  One workgroup goes through all that the bin has
  // each time, keys beyond kListed from memory: a row of 128256 equal logits takes 4400 us with top_k and 5300 with top_p, one at a temperature of 100 455.
  uint64_t last = 0;   // tokens of at least this key are kept
  constexpr int kPer = kMostParts / kThreads;
  double weights[kPer];
  uint32_t listed[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const uint32_t of = tid * kPer + i;
    weights[i] = 0., listed[i] = 0;
    if constexpr (WHOLE) {
      if (of == 0) weights[i] = kept, lds_more[of] = 0;
    } else if (of < a.parts) {
      weights[i] = __builtin_bit_cast(double, __hip_atomic_load((uint64_t*)&a.notes.kept[(uint64_t)r * a.parts + of], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
      if (open) weights[i] *= weight(logit_of_rank((uint32_t)(a.notes.keys[(uint64_t)r * a.parts + of] >> 32)));
      if (cuts) listed[i] = __hip_atomic_load(&a.notes.listed[(uint64_t)r * a.parts + of], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      lds_more[of] = 0;
    }
  }
  // (keys in the order of the parts: lds_upto[part] of them up to and with a part)
  auto read_key = [&](uint32_t at) {
    if constexpr (WHOLE) return __hip_atomic_load(&a.notes.list[(uint64_t)r * a.vocab + at], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    uint32_t low = 0, high = a.parts - 1;
    while (low < high) {
      const uint32_t middle = (low + high) / 2;
      if (lds_upto[middle] > at) high = middle;
      else low = middle + 1;
    }
    const uint32_t in_part = at - (low ? lds_upto[low - 1] : 0);
    return __hip_atomic_load(&a.notes.list[(uint64_t)r * a.vocab + low * kPart<CHUNKS> + in_part], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  };
  if (cuts && !WHOLE) {
    uint32_t mine = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) mine += listed[i];
    uint32_t in_wave = wave_upto(mine);
    if (lane == 63) lds_n[wave] = in_wave;
    __syncthreads();
    uint32_t before = in_wave - mine;
    for (uint32_t w = 0; w < kThreads / 64; ++w) {
      if (w < wave) before += lds_n[w];
      all_listed += lds_n[w];
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      before += listed[i];
      if (tid * kPer + i < a.parts) lds_upto[tid * kPer + i] = before;
    }
    __syncthreads();
    for (uint32_t i = tid; i < min(all_listed, kListed); i += kThreads) lds_keys[i] = read_key(i);
  }
  __syncthreads();
  auto listed_key = [&](uint32_t at) { return at < kListed ? lds_keys[at] : read_key(at); };
  auto logit_of = [&](uint64_t key) { return logit_of_rank((uint32_t)(key >> 32)); };
  if (cuts) {
    uint32_t left = all_listed, sub = 256;
    int shift = 64;   // bits of the key from here up are known
    auto candidate = [&](uint64_t key) {
      if (shift < 64 && (key ^ last) >> shift) return false;
      if (sub == 256) return true;
      const float d = distance_of(f, logit_of(key));
      return (uint32_t)fminf((d - (float)cut.bin) * 256.f, 255.f) == sub;
    };
    while (left > 64) {
      const bool by_place = sub == 256 && cut.bin != kBins - 1;
      if (tid < 256) lds_count[tid] = 0, lds_mass[tid] = 0;
      __syncthreads();
      for (uint32_t i = tid; i < all_listed; i += kThreads) {
        const uint64_t key = listed_key(i);
        if (!candidate(key)) continue;
        const float l = logit_of(key);
        // in falling order: the nearest place first, the largest digit first
        const uint32_t b = by_place ? (uint32_t)fminf((distance_of(f, l) - (float)cut.bin) * 256.f, 255.f) : 255 - ((uint32_t)(key >> (shift - 8)) & 255);
        atomicAdd(&lds_count[b], 1u);
        if (f.by_mass) atomicAdd((unsigned long long*)&lds_mass[b], (unsigned long long)mass_of(l));
      }
      __syncthreads();
      const uint32_t count[1] = {lds_count[tid]};
      const uint64_t mass[1] = {lds_mass[tid]};
      const uint32_t bin = cut.bin;
      const Cut in = find_cut<1>(count, mass, cut.above, cut.above_mass, f.k, f.by_mass, target, lds_n, lds_m, &lds_cut);
      left = lds_count[in.bin];
      cut = Cut{bin, in.above, in.above_mass};
      if (by_place) {
        sub = in.bin;
      } else {
        shift -= 8;
        last |= (uint64_t)(255 - in.bin) << shift;
        if (shift == 0) break;
      }
      __syncthreads();
    }
    // at most 64: a wavefront finds the smallest key that is kept (with all bits known there is one)
    if (tid == 0) lds_base = 0;
    __syncthreads();
    uint64_t mine = 0;
    for (uint32_t first = 0; first < all_listed; first += kThreads) {
      const uint64_t key = first + tid < all_listed ? listed_key(first + tid) : 0;
      if (first + tid < all_listed && candidate(key)) lds_mass[__hip_atomic_fetch_add(&lds_base, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP)] = key;
    }
    __syncthreads();
    if (wave == 0) {
      mine = lane < left ? lds_mass[lane] : 0;
      const uint64_t my_mass = lane < left && f.by_mass ? mass_of(logit_of(mine)) : 0;
      uint32_t before = cut.above;
      uint64_t mass_before = cut.above_mass;
      for (uint32_t j = 0; j < left; ++j) {
        const uint64_t other = of_lane(mine, j), its = of_lane(my_mass, j);
        if (other > mine) ++before, mass_before += its;
      }
      const bool stays = lane < left && (before == 0 || (before < f.k && (!f.by_mass || (double)mass_before < target)));
      uint64_t least_key = stays ? mine : ~0ull;
      least_key = ~wave_most(~least_key);
      if (lane == 0) slots[0] = least_key;
    }
    __syncthreads();
    last = slots[0];
    // kept tokens of the bin, added to their parts
    for (uint32_t i = tid; i < all_listed; i += kThreads) {
      const uint64_t key = listed_key(i);
      if (key < last) continue;
      const uint32_t token = ~(uint32_t)key;
      atomicAdd((unsigned long long*)&lds_more[token / kPart<CHUNKS>], (unsigned long long)(kept_weight(logit_of(key), token) * unit + 0.5));
    }
  }
  __syncthreads();

  // The part that the number falls into, then the token.
  double mine = 0.;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    if (tid * kPer + i < a.parts) weights[i] += (double)lds_more[tid * kPer + i] / unit;
    mine += weights[i];
  }
  // Sums up to a thread's, and of all: the wavefronts' in LDS.
  auto upto_of = [&](double v, double* all) {
    const double in_wave = wave_upto(v);
    __syncthreads();
    if (lane == 63) lds_sum[wave] = in_wave;
    __syncthreads();
    double before = 0.;
    *all = 0.;
    for (uint32_t w = 0; w < kThreads / 64; ++w) {
      if (w == wave) before = *all;
      *all += lds_sum[w];
    }
    return before + in_wave;
  };
  double total, reached = 0.;
  uint32_t of = 0;
  bool beyond = false;   // beyond all: the last token
  if constexpr (WHOLE) {
    total = kept + (double)lds_more[0] / unit;
    if (tid == 0) lds_last = 0, lds_token = ~0u;
  }
  const double upto = WHOLE ? 0. : upto_of(mine, &total), place = (double)a.uniform[r] * total;
  if constexpr (!WHOLE) {
    if (tid == 0) lds_base = ~0u, lds_last = 0, lds_token = ~0u;
    __syncthreads();
    {
      double upto_here = upto - mine;
      uint32_t first_of = ~0u, last_of = 0;
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const uint32_t one = tid * kPer + i;
        upto_here += weights[i];
        const bool has = one < a.parts && weights[i] > 0.;
        last_of = has ? one : last_of;
        first_of = has && upto_here > place ? min(first_of, one) : first_of;
      }
      first_of = wave_least(first_of), last_of = wave_most(last_of);
      if (lane == 0) atomicMin(&lds_base, first_of), atomicMax(&lds_last, last_of);
    }
    __syncthreads();
    of = lds_base != ~0u ? lds_base : lds_last, beyond = lds_base == ~0u;
    if (tid == of / kPer) {
      double before = upto - mine;
      for (int i = 0; i < kPer; ++i)
        if ((uint32_t)(tid * kPer + i) < of) before += weights[i];
      lds_share = before;
    }
    __syncthreads();
    reached = lds_share;
  }
  // (a thread takes neighbouring tokens here; from the caches, unless it has them)
  const uint32_t at0 = of * kPart<CHUNKS> + 4 * CHUNKS * tid;
  double own = 0.;
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) {
    if constexpr (!WHOLE) four_of(row, at0 + 4 * c, a.vocab, v[c]);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t i = at0 + 4 * c + j;
      const double one = WHOLE ? w[c][j] : kept_weight(v[c][j], i);
      w[c][j] = ((i < a.vocab) & (key_of(v[c][j], i) >= last)) ? one : 0.;
      own += w[c][j];
    }
  }
  double all_here;
  double here = reached + upto_of(own, &all_here) - own;
  uint32_t last_kept = 0, mine_first = ~0u;   // (a token's number and one; a token)
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      here += w[c][j];
      last_kept = w[c][j] > 0. ? at0 + 4 * c + j + 1 : last_kept;
      mine_first = w[c][j] > 0. && here > place ? min(mine_first, at0 + 4 * c + j) : mine_first;
    }
  mine_first = wave_least(beyond ? ~0u : mine_first), last_kept = wave_most(last_kept);
  if (lane == 0) atomicMin(&lds_token, mine_first), atomicMax(&lds_last, last_kept + kMostVocab);   // (above every part's number)
  __syncthreads();
  if (tid == 0) {
    const uint32_t token = lds_token != ~0u ? lds_token : lds_last - kMostVocab - 1;
    a.tokens[r] = (int32_t)token;
    if (a.probs) a.probs[r] = (float)(weight(logit_of_rank(rank_of(row[token]))) / total);
  }
}

struct Layout {
  uint64_t keys, kept, mass, count, listed, list, done, bytes;   // offsets
  uint32_t parts;
  bool whole, many;   // whole: a row is one workgroup's
};

int check_sample(const std::string& who, const tq_sample_args* a, Layout* l) {
  if (!a) return refuse(TQ_E_INVALID_ARG, who + ": null argument");
  if (a->vocab == 0 || a->vocab > kMostVocab) return refuse(TQ_E_UNSUPPORTED, who + ": vocab must be in 1..2^20");
  if (a->rows > 65535) return refuse(TQ_E_UNSUPPORTED, who + ": more than 65535 rows");
  if (a->logits_stride && a->logits_stride < a->vocab) return refuse(TQ_E_INVALID_ARG, who + ": logits_stride is smaller than a row");
  auto place = [&](uint64_t n) {
    const uint64_t at = (l->bytes + 255) / 256 * 256;
    l->bytes = at + n;
    return at;
  };
  // a row of one workgroup needs no launches ahead, but its weights are all behind each other: 16 rows with filters of 2048 logits 9.1 us in place of 18.7, of 4096 12.4 in place of 19.1, of 8192 19.7 in place of
  // 19.4; without filters 6.4 in place of 12.8, 7.1 and 12.8, 11.6 and 12.5; 1024 rows of 8192, whose threads need too many registers, 76 and 67, without filters 44 and 32
  l->whole = a->vocab <= kPart<4>;
  l->many = (uint64_t)a->rows * ((a->vocab + kPart<kFew> - 1) / kPart<kFew>) > 1024;
  const uint32_t part = l->whole ? kPart<4> : l->many ? kPart<kMany> : kPart<kFew>;
  l->parts = (a->vocab + part - 1) / part;
  l->bytes = 16;   // (a workspace is there in any case)
  const bool lists = a->top_k || a->top_p;
  if (l->whole) {
    // (a row of one workgroup leaves itself nothing but the keys that LDS has no room for)
    if (lists && a->vocab > kListed) l->list = place((uint64_t)a->rows * a->vocab * 8);
    return TQ_OK;
  }
  l->keys = place((uint64_t)a->rows * l->parts * 8);
  l->kept = place((uint64_t)a->rows * l->parts * 8);
  l->mass = place((uint64_t)a->rows * kBins * 8);
  l->count = place((uint64_t)a->rows * kBins * 4);
  l->listed = place((uint64_t)a->rows * l->parts * 4);
  l->done = place((uint64_t)a->rows * kApart * 4);
  if (lists) l->list = place((uint64_t)a->rows * a->vocab * 8);
  return TQ_OK;
}

int sample(const tq_sample_args* a, void* stream) {
  const std::string who = "tq_sample";
  Layout l{};
  if (int rc = check_sample(who, a, &l)) return rc;
  if (a->rows == 0) return TQ_OK;
  if (!a->logits || !a->uniform || !a->tokens || !a->workspace) return refuse(TQ_E_INVALID_ARG, who + ": null pointer");
  for (const void* p : {(const void*)a->logits, (const void*)a->temperature, (const void*)a->top_p, (const void*)a->min_p, (const void*)a->uniform, (const void*)a->top_k,
                        (const void*)a->tokens, (const void*)a->probs})
    if (!aligned_to(p, 4)) return refuse(TQ_E_INVALID_ARG, who + ": a pointer is not aligned to its type");
  if (!aligned_to(a->workspace, 16)) return refuse(TQ_E_INVALID_ARG, who + ": the workspace must be 16-byte aligned");
  if (a->workspace_bytes < l.bytes)
    return refuse(TQ_E_INVALID_ARG, who + ": the workspace has " + std::to_string(a->workspace_bytes) + " bytes, " + std::to_string(l.bytes) + " are needed");
  uint32_t bits = 62;
  while ((a->vocab >> (62 - bits)) > 0) --bits;   // a sum of vocab weights of at most 1 stays below 2^63
  char* ws = (char*)a->workspace;
  const Notes notes{(uint64_t*)(ws + l.keys), (uint64_t*)(ws + l.mass), (uint32_t*)(ws + l.count), (double*)(ws + l.kept), (uint32_t*)(ws + l.listed), (uint64_t*)(ws + l.list),
                    (uint32_t*)(ws + l.done)};
  const SampleView v{a->logits, a->temperature, a->top_p, a->min_p, a->uniform, a->top_k, a->tokens, a->probs, notes, a->logits_stride ? a->logits_stride : a->vocab, a->rows, a->vocab,
                     l.parts, bits};
  hipStream_t st = (hipStream_t)stream;
  auto go = [&](auto chunks) {
    constexpr int kChunks = decltype(chunks)::value;
    hipLaunchKernelGGL(k_sample_first<kChunks>, dim3(l.parts, a->rows), dim3(kThreads), 0, st, v);
    if (a->top_k || a->top_p) {
      // a workgroup per compute unit before a thread takes more than two tokens
      const uint32_t small = (a->vocab + 2 * kBinThreads - 1) / (2 * kBinThreads), large = (a->vocab + 8 * kBinThreads - 1) / (8 * kBinThreads);
      if ((uint64_t)small * a->rows <= 256) hipLaunchKernelGGL(k_sample_bins<2>, dim3(small, a->rows), dim3(kBinThreads), 0, st, v);
      else hipLaunchKernelGGL(k_sample_bins<8>, dim3(large, a->rows), dim3(kBinThreads), 0, st, v);
    }
    hipLaunchKernelGGL((k_sample_draw<kChunks, false>), dim3(a->rows, l.parts), dim3(kThreads), 0, st, v);
  };
  // (half as many tokens a thread where they are enough: 2048 logits 9.1 us, where 4096 take 12.4)
  auto whole = [&](auto chunks) { hipLaunchKernelGGL((k_sample_draw<decltype(chunks)::value, true>), dim3(a->rows), dim3(kThreads), 0, st, v); };
  if (l.whole && a->vocab <= kPart<2>) whole(std::integral_constant<int, 2>());
  else if (l.whole) whole(std::integral_constant<int, 4>());
  else if (l.many) go(std::integral_constant<int, kMany>());
  else go(std::integral_constant<int, kFew>());
  return launched("tq_sample");
}

}  // namespace
}  // namespace tq

extern "C" int tq_sample(const tq_sample_args* args, void* stream) {
  return tq::contained("tq_sample", [&] { return tq::sample(args, stream); });
}

extern "C" int tq_sample_workspace(const tq_sample_args* args, uint64_t* bytes) {
  return tq::contained("tq_sample_workspace", [&] {
    if (!bytes) return tq::refuse(TQ_E_INVALID_ARG, "tq_sample_workspace: null argument");
    tq::Layout l{};
    const int rc = tq::check_sample("tq_sample_workspace", args, &l);
    if (rc == TQ_OK) *bytes = l.bytes;
    return rc;
  });
}
