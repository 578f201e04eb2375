// Residual addition and root-mean-square norm (tq_add_rms_norm): h = residual + delta, y = h / sqrt(mean(h^2) + eps) * weight.
//
// Bound: device memory, or for few rows the chain load -> sum over the row -> store.  A workgroup takes a row, every thread
// keeps its values of h in registers between the sum and the output, so residual and delta are read once.  4096 rows of 8192, fp32 to bf16: 85 us,
// 5.5 TB/s read and written, to int8 80; of 2048: 23 us; one row of 2048 2.2 us.
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

// Four values at a time, at any address that their type allows: values i..i+3 of a row of n, fp32 or bf16; those beyond it are zero.  WHOLE:
// n is a multiple of 4.
template <bool WHOLE, bool BF16>
__device__ __forceinline__ void load_values(const void* row, uint32_t i, uint32_t n, float (&v)[4]) {
  if (WHOLE || i + 4 <= n) {
    if constexpr (BF16) {
      const u16x4_any d = *(const u16x4_any*)((const uint16_t*)row + i);
      v[0] = bf16_value(d.x), v[1] = bf16_value(d.y), v[2] = bf16_value(d.z), v[3] = bf16_value(d.w);
    } else {
      const f32x4_any d = *(const f32x4_any*)((const float*)row + i);
      v[0] = d.x, v[1] = d.y, v[2] = d.z, v[3] = d.w;
    }
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = i + k >= n ? 0.f : BF16 ? bf16_value(((const uint16_t*)row)[i + k]) : ((const float*)row)[i + k];
  }
}

template <bool WHOLE, bool BF16>
__device__ __forceinline__ void store_values(void* row, uint32_t i, uint32_t n, const float (&v)[4]) {
  if constexpr (BF16) {
    uint16_t* to = (uint16_t*)row + i;
    const uint32_t lo = pack_bf16(v[0], v[1]), hi = pack_bf16(v[2], v[3]);
    if (WHOLE || i + 4 <= n) {
      *(u16x4_any*)to = __builtin_bit_cast(u16x4_any, make_uint2(lo, hi));
    } else {
      if (i < n) to[0] = (uint16_t)lo;
      if (i + 1 < n) to[1] = (uint16_t)(lo >> 16);
      if (i + 2 < n) to[2] = (uint16_t)hi;
    }
  } else {
    float* to = (float*)row + i;
    if (WHOLE || i + 4 <= n) {
      *(f32x4_any*)to = f32x4_any{v[0], v[1], v[2], v[3]};
    } else {
#pragma unroll
      for (int k = 0; k < 3; ++k)
        if (i + k < n) to[k] = v[k];
    }
  }
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

// CHUNKS pieces of four values per thread (0: any number, read again for the output).
template <int CHUNKS, bool WHOLE, bool RES16, bool W16, bool OUT8>
__global__ __launch_bounds__(1024) void k_add_rms_norm(NormView a) {
  __shared__ float sums[16], tops[16];
  const uint64_t r = blockIdx.x;
  const char* res = (const char*)a.residual + r * a.residual_stride * (RES16 ? 2 : 4);
  const float* delta = a.delta ? a.delta + r * a.delta_stride : nullptr;
  char* res_out = a.residual_out ? (char*)a.residual_out + r * a.residual_out_stride * (RES16 ? 2 : 4) : nullptr;
  const uint32_t step = blockDim.x * 4;
  constexpr int KEEP = CHUNKS ? CHUNKS : 1;
  float h[KEEP][4], w[KEEP][4];
  auto sum_of = [&](uint32_t i, float (&x)[4]) {
    load_values<WHOLE, RES16>(res, i, a.cols, x);
    if (delta) {
      float d[4];
      load_values<WHOLE, false>(delta, i, a.cols, d);
#pragma unroll
      for (int k = 0; k < 4; ++k) x[k] += d[k];
    }
  };
  const float share = 1.f / (float)a.cols;   // of a value in the mean, taken before it is squared: a sum of squares overflows sooner
  float square = 0.f;
  if constexpr (CHUNKS) {
    // All of the row is requested before any of it is used, the weights too (4096 x 2999 43 -> 40 us, a bf16 residual of 4096 x 8192
    // 66 -> 61); in place of values beyond the row, its first ones.
    float d[CHUNKS][4] = {};
    auto place = [&](int c) {
      const uint32_t i = threadIdx.x * 4 + c * step;
      return WHOLE && i >= a.cols ? 0 : i;
    };
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) load_values<WHOLE, RES16>(res, place(c), a.cols, h[c]);
    if (delta) {
#pragma unroll
      for (int c = 0; c < CHUNKS; ++c) load_values<WHOLE, false>(delta, place(c), a.cols, d[c]);
    }
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) load_values<WHOLE, W16>(a.weight, place(c), a.cols, w[c]);
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
      const uint32_t i = threadIdx.x * 4 + c * step;
      if (i < a.cols) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          h[c][k] += d[c][k];
          square = fmaf(h[c][k] * share, h[c][k], square);
        }
        if (res_out) store_values<WHOLE, RES16>(res_out, i, a.cols, h[c]);
      }
    }
  } else {
    for (uint32_t i = threadIdx.x * 4; i < a.cols; i += step) {
      sum_of(i, h[0]);
#pragma unroll
      for (int k = 0; k < 4; ++k) square = fmaf(h[0][k] * share, h[0][k], square);
    }
  }
  square = over_waves(group_sum<64>(square), sums, [](float x, float y) { return x + y; });
  const float inv = 1.f / sqrtf(square + a.eps);
  auto normed = [&](uint32_t i, float (&x)[4], float (&w)[4]) {
    if (!CHUNKS) load_values<WHOLE, W16>(a.weight, i, a.cols, w);
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = x[k] * inv * w[k];
  };
  float scale = 0.f;
  if constexpr (OUT8) {
    float top = 0.f;
    auto see = [&](uint32_t i, float (&x)[4], float (&w)[4]) {
      normed(i, x, w);
#pragma unroll
      for (int k = 0; k < 4; ++k) top = max_or_nan(top, fabsf(x[k]));
    };
    if constexpr (CHUNKS) {
#pragma unroll
      for (int c = 0; c < CHUNKS; ++c) {
        const uint32_t i = threadIdx.x * 4 + c * step;
        if (i < a.cols) see(i, h[c], w[c]);
      }
    } else {
      for (uint32_t i = threadIdx.x * 4; i < a.cols; i += step) {
        sum_of(i, h[0]);
        see(i, h[0], w[0]);
      }
    }
    top = over_waves(wave_max_or_nan(top), tops, [](float x, float y) { return max_or_nan(x, y); });
    scale = scale_of(top);
    if (threadIdx.x == 0) a.out_scale[r] = scale;
  }
  auto put = [&](uint32_t i, float (&x)[4]) {
    if constexpr (OUT8) {
      int8_t* out = (int8_t*)a.out + r * a.out_stride + i;
      const uint32_t bytes = (uint32_t)(quantized(x[0], scale) & 255) | (uint32_t)(quantized(x[1], scale) & 255) << 8 |
                             (uint32_t)(quantized(x[2], scale) & 255) << 16 | (uint32_t)quantized(x[3], scale) << 24;
      if (WHOLE || i + 4 <= a.cols) {
        *(u32_any*)out = bytes;
      } else {
#pragma unroll
        for (int k = 0; k < 3; ++k)
          if (i + k < a.cols) out[k] = (int8_t)(bytes >> (8 * k));
      }
    } else {
      store_values<WHOLE, true>((uint16_t*)a.out + r * a.out_stride, i, a.cols, x);
    }
  };
  if constexpr (CHUNKS) {
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
      const uint32_t i = threadIdx.x * 4 + c * step;
      if (i < a.cols) {
        if constexpr (!OUT8) normed(i, h[c], w[c]);
        put(i, h[c]);
      }
    }
  } else {
    for (uint32_t i = threadIdx.x * 4; i < a.cols; i += step) {   // (residual_out may be residual: it is written after its last use)
      sum_of(i, h[0]);
      if (res_out) store_values<WHOLE, RES16>(res_out, i, a.cols, h[0]);
      normed(i, h[0], w[0]);
      put(i, h[0]);
    }
  }
}

template <int CHUNKS, bool WHOLE>
void launch_norm(const NormView& v, uint32_t threads, bool res16, bool w16, bool out8, hipStream_t stream) {
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(v.rows), dim3(threads), 0, stream, v); };
  if (res16) {
    if (w16) out8 ? go(k_add_rms_norm<CHUNKS, WHOLE, true, true, true>) : go(k_add_rms_norm<CHUNKS, WHOLE, true, true, false>);
    else out8 ? go(k_add_rms_norm<CHUNKS, WHOLE, true, false, true>) : go(k_add_rms_norm<CHUNKS, WHOLE, true, false, false>);
  } else {
    if (w16) out8 ? go(k_add_rms_norm<CHUNKS, WHOLE, false, true, true>) : go(k_add_rms_norm<CHUNKS, WHOLE, false, true, false>);
    else out8 ? go(k_add_rms_norm<CHUNKS, WHOLE, false, false, true>) : go(k_add_rms_norm<CHUNKS, WHOLE, false, false, false>);
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
  const uint32_t pieces = (a->cols + 3) / 4;
  const uint32_t chunks = pieces > 8192 ? 0 : pieces > 4096 ? 8 : pieces > 2048 ? 4 : pieces > 1024 ? 2 : 1;
  const uint32_t threads = chunks && chunks < 8 ? ((pieces + chunks - 1) / chunks + 63) / 64 * 64 : 1024;
  if ((uint64_t)a->rows * threads > 0xFFFFFFFFu) return refuse(TQ_E_UNSUPPORTED, who + ": too many rows for one launch");
  hipStream_t s = (hipStream_t)stream;
  auto go = [&](auto whole) {
    constexpr bool W = decltype(whole)::value;
    if (chunks == 1) launch_norm<1, W>(v, threads, res16, w16, out8, s);
    else if (chunks == 2) launch_norm<2, W>(v, threads, res16, w16, out8, s);
    else if (chunks == 4) launch_norm<4, W>(v, threads, res16, w16, out8, s);
    else if (chunks == 8) launch_norm<8, W>(v, threads, res16, w16, out8, s);
    else launch_norm<0, W>(v, threads, res16, w16, out8, s);
  };
  a->cols % 4 ? go(std::false_type()) : go(std::true_type());
  return launched("tq_add_rms_norm");
}

}  // namespace
}  // namespace tq

extern "C" int tq_add_rms_norm(const tq_norm_args* args, void* stream) {
  return tq::contained("tq_add_rms_norm", [&] { return tq::add_rms_norm(args, stream); });
}
