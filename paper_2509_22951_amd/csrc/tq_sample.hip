// One token per row, drawn from its logits (tq_sample).
#include <algorithm>

#include "tq_cache_view.h"

namespace tq {
namespace {

constexpr uint32_t kMostVocab = 1u << 20, kSampleThreads = 1024;

struct SampleView {
  const float* logits;
  const float *temperature, *top_p, *min_p, *uniform;
  const int32_t* top_k;
  int32_t* tokens;
  float* probs;
  uint64_t stride;
  uint32_t rows, vocab, mass_bits;   // weights are summed in units of 2^-mass_bits where the order of summation is not fixed
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

// A workgroup per row.  Bound: one compute unit reads the row once per digit.
__global__ __launch_bounds__(kSampleThreads) void k_sample(SampleView a) {
  __shared__ uint64_t lds_key[kSampleThreads / 64], lds_mass[256];
  __shared__ uint32_t lds_count[256];
  __shared__ double lds_sum[kSampleThreads];
  __shared__ uint64_t lds_above_mass;
  __shared__ uint32_t lds_above, lds_digit;
  const uint32_t r = blockIdx.x, tid = threadIdx.x, vocab = a.vocab;
  const float* row = a.logits + (uint64_t)r * a.stride;
  uint64_t best = 0;
  for (uint32_t i = tid; i < vocab; i += kSampleThreads) best = max(best, key_of(row[i], i));
#pragma unroll
  for (int d = 1; d < 64; d *= 2) best = max(best, (uint64_t)__shfl_xor((unsigned long long)best, d));
  if (tid % 64 == 0) lds_key[tid / 64] = best;
  __syncthreads();
  best = lds_key[0];
  for (uint32_t w = 1; w < kSampleThreads / 64; ++w) best = max(best, lds_key[w]);
  const uint32_t first = ~(uint32_t)best;
  const float top = row[first], temperature = a.temperature ? a.temperature[r] : 1.f;
  if (!(top > -INFINITY) || !(temperature > 0.f)) {
    if (tid == 0) {
      a.tokens[r] = top > -INFINITY ? (int32_t)first : -1;
      if (a.probs) a.probs[r] = top > -INFINITY ? 1.f : 0.f;
    }
    return;
  }
  const Weigher weight{(double)top, (double)temperature};
  const float want_p = a.top_p ? a.top_p[r] : 1.f, min_p = a.min_p ? a.min_p[r] : 0.f;
  const int32_t want_k = a.top_k ? a.top_k[r] : 0;
  const uint32_t k = want_k > 0 ? min((uint32_t)want_k, vocab) : vocab;
  const bool by_mass = want_p < 1.f;
  const double unit = (double)(1ull << a.mass_bits);
  auto mass_of = [&](float l) { return (uint64_t)(weight(l) * unit + 0.5); };
  uint64_t cut = 0;   // tokens of at least this key are kept
  if (by_mass || k < vocab) {
    if (tid == 0) lds_above = 0, lds_above_mass = 0;
    double target = 0.;
    for (int shift = 56; shift >= 0; shift -= 8) {
      __syncthreads();
      for (uint32_t b = tid; b < 256; b += kSampleThreads) lds_count[b] = 0, lds_mass[b] = 0;
      __syncthreads();
      for (uint32_t i = tid; i < vocab; i += kSampleThreads) {
        const uint64_t key = key_of(row[i], i);
        if (shift < 56 && (key ^ cut) >> (shift + 8)) continue;
        const uint32_t b = (uint32_t)(key >> shift) & 255;
        atomicAdd(&lds_count[b], 1u);
        if (by_mass) atomicAdd((unsigned long long*)&lds_mass[b], (unsigned long long)mass_of(row[i]));
      }
      __syncthreads();
      if (shift == 56) {
        uint64_t total = 0;
        for (uint32_t b = 0; b < 256; ++b) total += lds_mass[b];
        target = (double)want_p * (double)total;
      }
      if (tid == 0) {   // the bin in which the last token lies that is kept
        uint32_t above = lds_above, last = 0;
        uint64_t mass = lds_above_mass;
        for (int b = 255; b >= 0; --b) {
          if (!lds_count[b]) continue;
          const bool begins = above == 0 || (above < k && (!by_mass || (double)mass < target));
          if (!begins) break;
          last = b, lds_above = above, lds_above_mass = mass;
          above += lds_count[b], mass += lds_mass[b];
        }
        lds_digit = last;
      }
      __syncthreads();
      cut |= (uint64_t)lds_digit << shift;
    }
  }
  auto kept = [&](float l, uint32_t i) {
    const uint64_t key = key_of(l, i);
    if (key < cut) return 0.;
    const double w = weight(l);
    return key == best || !(w < (double)min_p) ? w : 0.;
  };
  const uint32_t per = (vocab + kSampleThreads - 1) / kSampleThreads, begin = min(tid * per, vocab), end = min(begin + per, vocab);
  double sum = 0.;
  for (uint32_t i = begin; i < end; ++i) sum += kept(row[i], i);
  lds_sum[tid] = sum;
  __syncthreads();
  if (tid == 0) {
    double total = 0.;
    for (uint32_t i = 0; i < kSampleThreads; ++i) total += lds_sum[i];
    const double place = (double)a.uniform[r] * total;
    double upto = 0.;
    uint32_t token = first;
    double share = 0.;
    bool found = false;
    for (uint32_t t = 0; t < kSampleThreads && !found; ++t) {
      const double next = upto + lds_sum[t];
      if (lds_sum[t] > 0. && next > place) {
        for (uint32_t i = t * per; i < min(t * per + per, vocab); ++i) {
          const double w = kept(row[i], i);
          if (!(w > 0.)) continue;
          upto += w, token = i, share = w;
          if (upto > place) break;
        }
        found = true;
      }
      upto = next;
    }
    if (!found) {   // beyond all of them: the last one
      for (uint32_t i = 0; i < vocab; ++i) {
        const double w = kept(row[i], i);
        if (w > 0.) token = i, share = w;
      }
    }
    a.tokens[r] = (int32_t)token;
    if (a.probs) a.probs[r] = (float)(share / total);
  }
}

int check_sample(const std::string& who, const tq_sample_args* a, uint64_t* bytes) {
  if (!a) return refuse(TQ_E_INVALID_ARG, who + ": null argument");
  if (a->vocab == 0 || a->vocab > kMostVocab) return refuse(TQ_E_UNSUPPORTED, who + ": vocab must be in 1..2^20");
  if (a->rows > 65535) return refuse(TQ_E_UNSUPPORTED, who + ": more than 65535 rows");
  if (a->logits_stride && a->logits_stride < a->vocab) return refuse(TQ_E_INVALID_ARG, who + ": logits_stride is smaller than a row");
  *bytes = 256;
  return TQ_OK;
}

int sample(const tq_sample_args* a, void* stream) {
  const std::string who = "tq_sample";
  uint64_t bytes = 0;
  if (int rc = check_sample(who, a, &bytes)) return rc;
  if (a->rows == 0) return TQ_OK;
  if (!a->logits || !a->uniform || !a->tokens || !a->workspace) return refuse(TQ_E_INVALID_ARG, who + ": null pointer");
  for (const void* p : {(const void*)a->logits, (const void*)a->temperature, (const void*)a->top_p, (const void*)a->min_p, (const void*)a->uniform, (const void*)a->top_k,
                        (const void*)a->tokens, (const void*)a->probs})
    if (!aligned_to(p, 4)) return refuse(TQ_E_INVALID_ARG, who + ": a pointer is not aligned to its type");
  if (!aligned_to(a->workspace, 16)) return refuse(TQ_E_INVALID_ARG, who + ": the workspace must be 16-byte aligned");
  if (a->workspace_bytes < bytes)
    return refuse(TQ_E_INVALID_ARG, who + ": the workspace has " + std::to_string(a->workspace_bytes) + " bytes, " + std::to_string(bytes) + " are needed");
  uint32_t bits = 62;
  while ((a->vocab >> (62 - bits)) > 0) --bits;   // a sum of vocab weights of at most 1 stays below 2^63
  const SampleView v{a->logits, a->temperature, a->top_p, a->min_p, a->uniform, a->top_k, a->tokens, a->probs, a->logits_stride ? a->logits_stride : a->vocab, a->rows, a->vocab, bits};
  hipLaunchKernelGGL(k_sample, dim3(a->rows), dim3(kSampleThreads), 0, (hipStream_t)stream, v);
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
    return tq::check_sample("tq_sample_workspace", args, bytes);
  });
}
