// One token per row, drawn from its logits (tq_sample).
#include <algorithm>

#include "tq_cache_view.h"

namespace tq {
namespace {

constexpr uint32_t kMostVocab = 1u << 20, kThreads = 256, kPart = 8 * kThreads;   // kPart: logits of a workgroup
constexpr uint32_t kBinThreads = 1024, kBinPart = 8 * kBinThreads, kBins = 2048, kBinsPerUnit = 32, kListed = 2048;   // bins of (largest - logit) / temperature; keys held in LDS

// What the launches leave each other, for every row.
struct Notes {
  uint64_t* keys;      // [row][part]: the first token's key
  uint64_t* mass;      // [row][kBins]: weights of a bin
  uint32_t* count;     // [row][kBins]: tokens of a bin
  double* kept;        // [row][part]: weight of what is kept beyond doubt
  uint32_t* listed;    // [row][2]: tokens in the list, workgroups that are done
  uint32_t* list;      // [row][vocab]: tokens of the bin that the cut lies in
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

struct Weigher {
  double top, temperature;
  __device__ __forceinline__ double operator()(float l) const {
    if (!(l > -INFINITY)) return 0.;
    if (top == INFINITY) return l == INFINITY ? 1. : 0.;
    return exp(((double)l - top) / temperature);
  }
};

// How a row is to be drawn from.
struct Filter {
  float top, temperature, p, least;
  uint32_t first, k;
  bool drawn, by_rank, by_mass;   // drawn: not merely the first token; by_rank, by_mass: top_k or top_p leaves something out
};

__device__ __forceinline__ uint64_t wave_max(uint64_t v) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) v = max(v, (uint64_t)__shfl_xor((unsigned long long)v, d));
  return v;
}
template <typename T>
__device__ __forceinline__ T wave_sum(T v) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
  return v;
}
// Sums over a wavefront's lanes up to and with each, in the same order every time.
template <typename T>
__device__ __forceinline__ T wave_upto(T v) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const T other = __shfl_up(v, d);
    if ((threadIdx.x & 63) >= (uint32_t)d) v += other;
  }
  return v;
}

// The first token's key of the row, from the parts' (by all threads; slots: one per wavefront).
__device__ __forceinline__ Filter filter_of(const SampleView& a, uint32_t r, uint64_t* slots) {
  uint64_t best = 0;
  for (uint32_t i = threadIdx.x; i < a.parts; i += blockDim.x) best = max(best, a.notes.keys[(uint64_t)r * a.parts + i]);
  best = wave_max(best);
  if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = best;
  __syncthreads();
  best = slots[0];
  for (uint32_t w = 1; w < blockDim.x / 64; ++w) best = max(best, slots[w]);
  Filter f;
  f.first = ~(uint32_t)best;
  f.top = a.logits[r * a.stride + f.first];
  f.temperature = a.temperature ? a.temperature[r] : 1.f;
  f.p = a.top_p ? a.top_p[r] : 1.f, f.least = a.min_p ? a.min_p[r] : 0.f;
  const int32_t k = a.top_k ? a.top_k[r] : 0;
  f.k = k > 0 ? min((uint32_t)k, a.vocab) : a.vocab;
  f.drawn = f.top > -INFINITY && f.temperature > 0.f;
  f.by_rank = f.k < a.vocab, f.by_mass = f.p < 1.f;
  return f;
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
  if (l == f.top) return 0.f;
  return l > -INFINITY ? (f.top - l) / f.temperature * (float)kBinsPerUnit : INFINITY;
}
__device__ __forceinline__ uint32_t bin_of(float distance) { return distance < (float)(kBins - 1) ? (uint32_t)distance : kBins - 1; }

// First launch: the first token of every part; bins and counters are cleared for the next ones.
__global__ __launch_bounds__(kThreads) void k_sample_first(SampleView a) {
  __shared__ uint64_t slots[kThreads / 64];
  const uint32_t part = blockIdx.x, r = blockIdx.y, tid = threadIdx.x;
  const float* row = a.logits + r * a.stride;
  float v[2][4];
#pragma unroll
  for (int c = 0; c < 2; ++c) four_of(row, part * kPart + c * (kPart / 2) + 4 * tid, a.vocab, v[c]);
  for (uint32_t i = part * kThreads + tid; i < kBins; i += a.parts * kThreads) a.notes.mass[(uint64_t)r * kBins + i] = 0, a.notes.count[(uint64_t)r * kBins + i] = 0;
  if (part == 0 && tid < 2) a.notes.listed[2 * r + tid] = 0;
  uint64_t best = 0;
#pragma unroll
  for (int c = 0; c < 2; ++c)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t i = part * kPart + c * (kPart / 2) + 4 * tid + j;
      if (i < a.vocab) best = max(best, key_of(v[c][j], i));
    }
  best = wave_max(best);
  if ((tid & 63) == 0) slots[tid >> 6] = best;
  __syncthreads();
  if (tid == 0) {
    for (uint32_t w = 1; w < kThreads / 64; ++w) best = max(best, slots[w]);
    a.notes.keys[(uint64_t)r * a.parts + part] = best;
  }
}

// Second launch, for rows with top_k or top_p: tokens and weights of every bin.
__global__ __launch_bounds__(kBinThreads) void k_sample_bins(SampleView a) {
  __shared__ uint64_t slots[kBinThreads / 64], lds_mass[kBins];
  __shared__ uint32_t lds_count[kBins];
  const uint32_t r = blockIdx.y, tid = threadIdx.x;
  const float* row = a.logits + r * a.stride;
  float v[2][4];
#pragma unroll
  for (int c = 0; c < 2; ++c) four_of(row, blockIdx.x * kBinPart + c * (kBinPart / 2) + 4 * tid, a.vocab, v[c]);
  for (uint32_t b = tid; b < kBins; b += kBinThreads) lds_mass[b] = 0, lds_count[b] = 0;
  const Filter f = filter_of(a, r, slots);
  if (!f.drawn || (!f.by_rank && !f.by_mass)) return;
  const Weigher weight{(double)f.top, (double)f.temperature};
  const double unit = (double)(1ull << a.mass_bits);
#pragma unroll
  for (int c = 0; c < 2; ++c)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t i = blockIdx.x * kBinPart + c * (kBinPart / 2) + 4 * tid + j;
      if (i >= a.vocab) continue;
      const uint32_t b = bin_of(distance_of(f, v[c][j]));
      atomicAdd(&lds_count[b], 1u);
      if (f.by_mass) atomicAdd((unsigned long long*)&lds_mass[b], (unsigned long long)(weight(v[c][j]) * unit + 0.5));
    }
  __syncthreads();
  for (uint32_t b = tid; b < kBins; b += kBinThreads)
    if (lds_count[b]) {
      atomicAdd(&a.notes.count[(uint64_t)r * kBins + b], lds_count[b]);
      if (f.by_mass) atomicAdd((unsigned long long*)&a.notes.mass[(uint64_t)r * kBins + b], (unsigned long long)lds_mass[b]);
    }
}

// The place in an order of bins, tokens and weights of a thread's neighbouring ones given, in which the last token lies that is kept: its first bin where a cut has come, or the
// last one that has tokens.  -> through LDS, by all threads.
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
  const uint64_t m_upto = wave_upto((unsigned long long)m);
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

// Third launch: the weight of what is kept in every part, and the tokens of the bin that the cut lies in; the last workgroup of a row finds the cut and draws.
//
// Bound: the three launches; 64 rows of 128256 logits are read three times, twice of it from the caches.
__global__ __launch_bounds__(kThreads) void k_sample_draw(SampleView a) {
  __shared__ uint64_t slots[kThreads / 64], lds_m[kThreads / 64], lds_keys[kListed], lds_mass[256], lds_more[kMostVocab / kPart];
  __shared__ uint32_t lds_n[kThreads / 64], lds_count[256], lds_base, lds_done, lds_token, lds_last;
  __shared__ double lds_sum[kThreads / 64], lds_share;
  __shared__ Cut lds_cut;
  const uint32_t part = blockIdx.x, r = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const float* row = a.logits + r * a.stride;
  float v[2][4];
#pragma unroll
  for (int c = 0; c < 2; ++c) four_of(row, part * kPart + c * (kPart / 2) + 4 * tid, a.vocab, v[c]);
  const Filter f = filter_of(a, r, slots);
  if (!f.drawn) {
    if (part == 0 && tid == 0) {
      a.tokens[r] = f.top > -INFINITY ? (int32_t)f.first : -1;
      if (a.probs) a.probs[r] = f.top > -INFINITY ? 1.f : 0.f;
    }
    return;
  }
  const Weigher weight{(double)f.top, (double)f.temperature};
  const double unit = (double)(1ull << a.mass_bits), least = (double)f.least;
  auto mass_of = [&](float l) { return (uint64_t)(weight(l) * unit + 0.5); };
  const bool cuts = f.by_rank || f.by_mass;
  Cut cut{kBins, 0, 0};
  double target = 0.;
  if (cuts) {
    constexpr int kPer = kBins / kThreads;
    uint32_t count[kPer];
    uint64_t mass[kPer], all = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      count[i] = a.notes.count[(uint64_t)r * kBins + tid * kPer + i], mass[i] = f.by_mass ? a.notes.mass[(uint64_t)r * kBins + tid * kPer + i] : 0;
      all += mass[i];
    }
    all = wave_sum((unsigned long long)all);
    if (lane == 0) lds_m[wave] = all;
    __syncthreads();
    all = 0;
    for (uint32_t w = 0; w < kThreads / 64; ++w) all += lds_m[w];
    target = (double)f.p * (double)all;
    cut = find_cut<kPer>(count, mass, 0, 0, f.k, f.by_mass, target, lds_n, lds_m, &lds_cut);
  }
  auto kept_weight = [&](float l, uint32_t i) {   // of a token that no cut leaves out
    const double w = weight(l);
    return i == f.first || !(w < least) ? w : 0.;
  };

  // this part
  double sum = 0.;
  uint32_t n = 0;
#pragma unroll
  for (int c = 0; c < 2; ++c)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t i = part * kPart + c * (kPart / 2) + 4 * tid + j;
      if (i >= a.vocab) continue;
      const uint32_t b = cuts ? bin_of(distance_of(f, v[c][j])) : 0;
      if (b < cut.bin) sum += kept_weight(v[c][j], i);
      n += b == cut.bin;
    }
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
  if (tid == 0) {
    double all = 0.;
    for (uint32_t w = 0; w < kThreads / 64; ++w) all += lds_sum[w];
    __hip_atomic_store((uint64_t*)&a.notes.kept[(uint64_t)r * a.parts + part], __builtin_bit_cast(uint64_t, all), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    lds_base = all_n ? __hip_atomic_fetch_add(&a.notes.listed[2 * r], all_n, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0;
  }
  __syncthreads();
  if (all_n) {
    at += lds_base;
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t i = part * kPart + c * (kPart / 2) + 4 * tid + j;
        if (i < a.vocab && bin_of(distance_of(f, v[c][j])) == cut.bin) __hip_atomic_store(&a.notes.list[(uint64_t)r * a.vocab + at++], i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      }
  }
  // the stores have reached the level that the device shares; the last workgroup goes on with all of the row
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (tid == 0) lds_done = __hip_atomic_fetch_add(&a.notes.listed[2 * r + 1], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  if (lds_done != a.parts - 1) return;

  // The cut within the bin: narrowed by a 256th of the bin, then by 8 bits of the key at a time, until few enough are left to compare all with each other.
  uint64_t last = 0;   // tokens of at least this key are kept
  for (uint32_t i = tid; i < a.parts; i += kThreads) lds_more[i] = 0;
  const uint32_t all_listed = cuts ? __hip_atomic_load(&a.notes.listed[2 * r], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0;
  auto read_key = [&](uint32_t at) {
    const uint32_t i = __hip_atomic_load(&a.notes.list[(uint64_t)r * a.vocab + at], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return key_of(row[i], i);
  };
  if (cuts) {
    for (uint32_t i = tid; i < min(all_listed, kListed); i += kThreads) lds_keys[i] = read_key(i);
    __syncthreads();
  }
  auto listed_key = [&](uint32_t at) { return at < kListed ? lds_keys[at] : read_key(at); };
  auto logit_of = [&](uint64_t key) { return row[~(uint32_t)key]; };
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
        const uint64_t other = (uint64_t)__shfl((unsigned long long)mine, j), its = (uint64_t)__shfl((unsigned long long)my_mass, j);
        if (other > mine) ++before, mass_before += its;
      }
      const bool stays = lane < left && (before == 0 || (before < f.k && (!f.by_mass || (double)mass_before < target)));
      uint64_t least_key = stays ? mine : ~0ull;
#pragma unroll
      for (int d = 1; d < 64; d *= 2) least_key = min(least_key, (uint64_t)__shfl_xor((unsigned long long)least_key, d));
      if (lane == 0) slots[0] = least_key;
    }
    __syncthreads();
    last = slots[0];
    // kept tokens of the bin, added to their parts
    for (uint32_t i = tid; i < all_listed; i += kThreads) {
      const uint64_t key = listed_key(i);
      if (key < last) continue;
      const uint32_t token = ~(uint32_t)key;
      atomicAdd((unsigned long long*)&lds_more[token / kPart], (unsigned long long)(kept_weight(row[token], token) * unit + 0.5));
    }
  }
  __syncthreads();

  // The part that the number falls into, then the token.
  constexpr int kPer = kMostVocab / kPart / kThreads;
  double weights[kPer], mine = 0.;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const uint32_t of = tid * kPer + i;
    weights[i] = 0.;
    if (of < a.parts)
      weights[i] = __builtin_bit_cast(double, __hip_atomic_load((uint64_t*)&a.notes.kept[(uint64_t)r * a.parts + of], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)) + (double)lds_more[of] / unit;
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
  double total;
  const double upto = upto_of(mine, &total);
  const double place = (double)a.uniform[r] * total;
  if (tid == 0) lds_base = ~0u, lds_last = 0, lds_token = ~0u;
  __syncthreads();
  {
    double reached = upto - mine;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const uint32_t of = tid * kPer + i;
      reached += weights[i];
      if (of < a.parts && weights[i] > 0.) {
        atomicMax(&lds_last, of);
        if (reached > place) atomicMin(&lds_base, of);
      }
    }
  }
  __syncthreads();
  const uint32_t of = lds_base != ~0u ? lds_base : lds_last;
  const bool beyond = lds_base == ~0u;   // beyond all: the last token
  if (tid == of / kPer) {
    double before = upto - mine;
    for (int i = 0; i < kPer; ++i)
      if ((uint32_t)(tid * kPer + i) < of) before += weights[i];
    lds_share = before;
  }
  __syncthreads();
  double reached = lds_share;
  const uint32_t first = of * kPart;
  uint32_t last_kept = 0;   // (a token's number and one)
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    float x[4];
    double w[4], four = 0.;
    const uint32_t at0 = first + c * (kPart / 2) + 4 * tid;
    four_of(row, at0, a.vocab, x);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      w[j] = at0 + j < a.vocab && key_of(x[j], at0 + j) >= last ? kept_weight(x[j], at0 + j) : 0.;
      four += w[j];
    }
    double all;
    double here = reached + upto_of(four, &all) - four;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      here += w[j];
      if (w[j] > 0.) {
        last_kept = at0 + j + 1;
        if (!beyond && here > place) atomicMin(&lds_token, at0 + j);
      }
    }
    reached += all;
  }
  if (last_kept) atomicMax(&lds_last, last_kept + kMostVocab);   // (above every part's number)
  __syncthreads();
  if (tid == 0) {
    const uint32_t token = lds_token != ~0u ? lds_token : lds_last - kMostVocab - 1;
    a.tokens[r] = (int32_t)token;
    if (a.probs) a.probs[r] = (float)(weight(row[token]) / total);
  }
}

struct Layout {
  uint64_t keys, kept, mass, count, listed, list, bytes;   // offsets
  uint32_t parts;
};

int check_sample(const std::string& who, const tq_sample_args* a, Layout* l) {
  if (!a) return refuse(TQ_E_INVALID_ARG, who + ": null argument");
  if (a->vocab == 0 || a->vocab > kMostVocab) return refuse(TQ_E_UNSUPPORTED, who + ": vocab must be in 1..2^20");
  if (a->rows > 65535) return refuse(TQ_E_UNSUPPORTED, who + ": more than 65535 rows");
  if (a->logits_stride && a->logits_stride < a->vocab) return refuse(TQ_E_INVALID_ARG, who + ": logits_stride is smaller than a row");
  auto place = [&](uint64_t n) {
    const uint64_t at = l->bytes;
    l->bytes += (n + 255) / 256 * 256;
    return at;
  };
  l->parts = (a->vocab + kPart - 1) / kPart;
  l->bytes = 0;
  l->keys = place((uint64_t)a->rows * l->parts * 8);
  l->kept = place((uint64_t)a->rows * l->parts * 8);
  l->mass = place((uint64_t)a->rows * kBins * 8);
  l->count = place((uint64_t)a->rows * kBins * 4);
  l->listed = place((uint64_t)a->rows * 8);
  l->list = place((uint64_t)a->rows * a->vocab * 4);
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
  const Notes notes{(uint64_t*)(ws + l.keys), (uint64_t*)(ws + l.mass), (uint32_t*)(ws + l.count), (double*)(ws + l.kept), (uint32_t*)(ws + l.listed), (uint32_t*)(ws + l.list)};
  const SampleView v{a->logits, a->temperature, a->top_p, a->min_p, a->uniform, a->top_k, a->tokens, a->probs, notes, a->logits_stride ? a->logits_stride : a->vocab, a->rows, a->vocab,
                     l.parts, bits};
  hipStream_t st = (hipStream_t)stream;
  hipLaunchKernelGGL(k_sample_first, dim3(l.parts, a->rows), dim3(kThreads), 0, st, v);
  if (a->top_k || a->top_p) hipLaunchKernelGGL(k_sample_bins, dim3((a->vocab + kBinPart - 1) / kBinPart, a->rows), dim3(kBinThreads), 0, st, v);
  hipLaunchKernelGGL(k_sample_draw, dim3(l.parts, a->rows), dim3(kThreads), 0, st, v);
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
