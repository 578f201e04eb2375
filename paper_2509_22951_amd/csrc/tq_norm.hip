// Residual addition and root-mean-square norm (tq_add_rms_norm): h = residual + delta, y = h / sqrt(mean(h^2) + eps) * weight.
//
// Bound: device memory, or for few rows the chain load -> sum over the row -> store.  A workgroup takes a row, every thread
// keeps its values of h in registers between the sum and the output, so residual and delta are read once.
#include "tq_cache_view.h"

namespace tq {
namespace {

struct NormView {
  const void* residual;
  const float* delta;
  const void* weight;
  void *residual_out, *out;
  float* out_scale;
  uint64_t residual_stride, delta_stride, residual_out_stride, out_stride;
  uint32_t rows, cols;
  float eps;
};

// VEC values at element i (a multiple of VEC) of a row of fp32 or bf16.
template <int VEC, bool BF16>
__device__ __forceinline__ void load_values(const void* row, uint32_t i, float (&v)[VEC]) {
  if constexpr (VEC == 4 && BF16) {
    const uint2 d = *(const uint2*)((const uint16_t*)row + i);
    v[0] = bf16_value(d.x), v[1] = __uint_as_float(d.x & 0xFFFF0000u), v[2] = bf16_value(d.y), v[3] = __uint_as_float(d.y & 0xFFFF0000u);
  } else if constexpr (VEC == 4) {
    const float4 d = *(const float4*)((const float*)row + i);
    v[0] = d.x, v[1] = d.y, v[2] = d.z, v[3] = d.w;
  } else if constexpr (BF16) {
    v[0] = bf16_value(((const uint16_t*)row)[i]);
  } else {
    v[0] = ((const float*)row)[i];
  }
}

template <int VEC, bool BF16>
__device__ __forceinline__ void store_values(void* row, uint32_t i, const float (&v)[VEC]) {
  if constexpr (VEC == 4 && BF16)
    *(uint2*)((uint16_t*)row + i) = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
  else if constexpr (VEC == 4)
    *(float4*)((float*)row + i) = make_float4(v[0], v[1], v[2], v[3]);
  else if constexpr (BF16)
    ((uint16_t*)row)[i] = (uint16_t)pack_bf16(v[0], 0.f);
  else
    ((float*)row)[i] = v[0];
}

// One value of every wavefront -> the combined one in all threads.  slots: one per wavefront, unused since the last barrier.
template <typename F>
__device__ __forceinline__ float over_waves(float v, float* slots, F&& join) {
  if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = v;
  __syncthreads();
  float all = slots[0];
  for (uint32_t w = 1; w < blockDim.x / 64; ++w) all = join(all, slots[w]);
  return all;
}

__device__ __forceinline__ float wave_max_or_nan(float v) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) v = max_or_nan(v, __shfl_xor(v, d));
  return v;
}

// CHUNKS pieces of VEC values per thread (0: any number, read again for the output).
template <int VEC, int CHUNKS, bool RES16, bool W16, bool OUT8>
__global__ __launch_bounds__(1024) void k_add_rms_norm(NormView a) {
  __shared__ float sums[16], tops[16];
  const uint64_t r = blockIdx.x;
  const char* res = (const char*)a.residual + r * a.residual_stride * (RES16 ? 2 : 4);
  const float* delta = a.delta ? a.delta + r * a.delta_stride : nullptr;
  char* res_out = a.residual_out ? (char*)a.residual_out + r * a.residual_out_stride * (RES16 ? 2 : 4) : nullptr;
  const uint32_t step = blockDim.x * VEC;
  constexpr int KEEP = CHUNKS ? CHUNKS : 1;
  float h[KEEP][VEC];
  auto sum_of = [&](uint32_t i, float (&x)[VEC]) {
    load_values<VEC, RES16>(res, i, x);
    if (delta) {
      float d[VEC];
      load_values<VEC, false>(delta, i, d);
#pragma unroll
      for (int k = 0; k < VEC; ++k) x[k] += d[k];
    }
  };
  const float share = 1.f / (float)a.cols;   // of a value in the mean, taken before it is squared: a sum of squares overflows sooner
  float square = 0.f;
  auto take = [&](uint32_t i, float (&x)[VEC]) {
    sum_of(i, x);
#pragma unroll
    for (int k = 0; k < VEC; ++k) square = fmaf(x[k] * share, x[k], square);
    if (CHUNKS && res_out) store_values<VEC, RES16>(res_out, i, x);
  };
  if constexpr (CHUNKS) {
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
      const uint32_t i = threadIdx.x * VEC + c * step;
      if (i < a.cols) take(i, h[c]);
    }
  } else {
    for (uint32_t i = threadIdx.x * VEC; i < a.cols; i += step) take(i, h[0]);
  }
  square = over_waves(group_sum<64>(square), sums, [](float x, float y) { return x + y; });
  const float inv = 1.f / sqrtf(square + a.eps);
  auto normed = [&](uint32_t i, float (&x)[VEC]) {
    float w[VEC];
    load_values<VEC, W16>(a.weight, i, w);
#pragma unroll
    for (int k = 0; k < VEC; ++k) x[k] = x[k] * inv * w[k];
  };
  float scale = 0.f;
  if constexpr (OUT8) {
    float top = 0.f;
    auto see = [&](uint32_t i, float (&x)[VEC]) {
      normed(i, x);
#pragma unroll
      for (int k = 0; k < VEC; ++k) top = max_or_nan(top, fabsf(x[k]));
    };
    if constexpr (CHUNKS) {
#pragma unroll
      for (int c = 0; c < CHUNKS; ++c) {
        const uint32_t i = threadIdx.x * VEC + c * step;
        if (i < a.cols) see(i, h[c]);
      }
    } else {
      for (uint32_t i = threadIdx.x * VEC; i < a.cols; i += step) {
        sum_of(i, h[0]);
        see(i, h[0]);
      }
    }
    top = over_waves(wave_max_or_nan(top), tops, [](float x, float y) { return max_or_nan(x, y); });
    scale = scale_of(top);
    if (threadIdx.x == 0) a.out_scale[r] = scale;
  }
  auto put = [&](uint32_t i, float (&x)[VEC]) {
    if constexpr (OUT8) {
      int8_t* out = (int8_t*)a.out + r * a.out_stride + i;
      if constexpr (VEC == 4)
        *(uint32_t*)out = (uint32_t)(quantized(x[0], scale) & 255) | (uint32_t)(quantized(x[1], scale) & 255) << 8 |
                          (uint32_t)(quantized(x[2], scale) & 255) << 16 | (uint32_t)quantized(x[3], scale) << 24;
      else
        *out = (int8_t)quantized(x[0], scale);
    } else {
      store_values<VEC, true>((uint16_t*)a.out + r * a.out_stride, i, x);
    }
  };
  if constexpr (CHUNKS) {
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
      const uint32_t i = threadIdx.x * VEC + c * step;
      if (i < a.cols) {
        if constexpr (!OUT8) normed(i, h[c]);
        put(i, h[c]);
      }
    }
  } else {
    for (uint32_t i = threadIdx.x * VEC; i < a.cols; i += step) {   // (residual_out may be residual: it is written after its last use)
      sum_of(i, h[0]);
      if (res_out) store_values<VEC, RES16>(res_out, i, h[0]);
      normed(i, h[0]);
      put(i, h[0]);
    }
  }
}

template <int VEC, int CHUNKS>
void launch_norm(const NormView& v, uint32_t threads, bool res16, bool w16, bool out8, hipStream_t stream) {
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(v.rows), dim3(threads), 0, stream, v); };
  if (res16) {
    if (w16) out8 ? go(k_add_rms_norm<VEC, CHUNKS, true, true, true>) : go(k_add_rms_norm<VEC, CHUNKS, true, true, false>);
    else out8 ? go(k_add_rms_norm<VEC, CHUNKS, true, false, true>) : go(k_add_rms_norm<VEC, CHUNKS, true, false, false>);
  } else {
    if (w16) out8 ? go(k_add_rms_norm<VEC, CHUNKS, false, true, true>) : go(k_add_rms_norm<VEC, CHUNKS, false, true, false>);
    else out8 ? go(k_add_rms_norm<VEC, CHUNKS, false, false, true>) : go(k_add_rms_norm<VEC, CHUNKS, false, false, false>);
  }
}

int add_rms_norm(const tq_norm_args* a, void* stream) {
  const std::string who = "tq_add_rms_norm";
  if (!a) return refuse(TQ_E_INVALID_ARG, who + ": null argument");
  if (a->residual_type > TQ_FP32 || a->weight_type > TQ_FP32) return refuse(TQ_E_UNSUPPORTED, who + ": residual and weight are TQ_FP32 or TQ_BF16");
  if (a->out_type != TQ_BF16 && a->out_type != TQ_INT8) return refuse(TQ_E_UNSUPPORTED, who + ": out is TQ_BF16 or TQ_INT8");
  if (a->cols == 0 || a->cols > (1u << 20)) return refuse(TQ_E_UNSUPPORTED, who + ": cols must be in 1..2^20");
  if (a->rows == 0) return TQ_OK;
  if (a->rows > 0x7FFFFFFFu) return refuse(TQ_E_UNSUPPORTED, who + ": too many rows");
  const bool out8 = a->out_type == TQ_INT8, res16 = a->residual_type == TQ_BF16, w16 = a->weight_type == TQ_BF16;
  if (!a->residual || !a->weight || !a->out || (out8 && !a->out_scale)) return refuse(TQ_E_INVALID_ARG, who + ": null pointer");
  NormView v{a->residual, a->delta, a->weight, a->residual_out, a->out, a->out_scale,
             a->residual_stride ? a->residual_stride : a->cols, a->delta_stride ? a->delta_stride : a->cols,
             a->residual_out_stride ? a->residual_out_stride : a->cols, a->out_stride ? a->out_stride : a->cols, a->rows, a->cols, a->eps};
  if (v.residual_stride < a->cols || v.delta_stride < a->cols || v.residual_out_stride < a->cols || v.out_stride < a->cols)
    return refuse(TQ_E_INVALID_ARG, who + ": a stride is smaller than cols");
  if (a->residual_out == a->residual && v.residual_out_stride != v.residual_stride)
    return refuse(TQ_E_INVALID_ARG, who + ": residual_out is residual, with another stride");
  if (!(a->eps >= 0.f)) return refuse(TQ_E_INVALID_ARG, who + ": eps must not be negative");
  const size_t res_size = res16 ? 2 : 4, out_size = out8 ? 1 : 2;
  if (!aligned_to(a->residual, res_size) || !aligned_to(a->residual_out, res_size) || !aligned_to(a->delta, 4) ||
      !aligned_to(a->weight, w16 ? 2 : 4) || !aligned_to(a->out, out_size) || !aligned_to(a->out_scale, 4))
    return refuse(TQ_E_INVALID_ARG, who + ": a pointer is not aligned to its type");
  auto fours = [](const void* p, uint64_t stride, size_t size) { return stride % 4 == 0 && aligned_to(p, 4 * size); };
  const bool by4 = a->cols % 4 == 0 && fours(a->residual, v.residual_stride, res_size) && fours(a->delta, v.delta_stride, 4) &&
                   fours(a->residual_out, v.residual_out_stride, res_size) && fours(a->out, v.out_stride, out_size) && aligned_to(a->weight, w16 ? 8 : 16);
  const uint32_t pieces = a->cols / (by4 ? 4 : 1);
  const uint32_t chunks = pieces > 4096 ? 0 : pieces > 2048 ? 4 : pieces > 1024 ? 2 : 1;
  const uint32_t threads = chunks ? ((pieces + chunks - 1) / chunks + 63) / 64 * 64 : 1024;
  hipStream_t s = (hipStream_t)stream;
  if (by4) {
    if (chunks == 1) launch_norm<4, 1>(v, threads, res16, w16, out8, s);
    else if (chunks == 2) launch_norm<4, 2>(v, threads, res16, w16, out8, s);
    else if (chunks == 4) launch_norm<4, 4>(v, threads, res16, w16, out8, s);
    else launch_norm<4, 0>(v, threads, res16, w16, out8, s);
  } else {
    if (chunks == 1) launch_norm<1, 1>(v, threads, res16, w16, out8, s);
    else if (chunks == 2) launch_norm<1, 2>(v, threads, res16, w16, out8, s);
    else if (chunks == 4) launch_norm<1, 4>(v, threads, res16, w16, out8, s);
    else launch_norm<1, 0>(v, threads, res16, w16, out8, s);
  }
  return launched("tq_add_rms_norm");
}

}  // namespace
}  // namespace tq

extern "C" int tq_add_rms_norm(const tq_norm_args* args, void* stream) {
  return tq::contained("tq_add_rms_norm", [&] { return tq::add_rms_norm(args, stream); });
}
