// What the kernels between the products share: a paged cache as they see it, the checks of its description, small device helpers.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>
#include <new>
#include <string>

#include "../../include/tq.h"
#include "tq_format.h"

namespace tq {

// tq_cache with its defaults filled in.  Offsets of pages, heads and slots are in elements and pass 32 bits in a long cache.
struct CacheView {
  char *k, *v;
  float *k_scale, *v_scale;   // [page][head][slot]
  const int32_t* tables;
  float* scores;              // [seq][head][slot]
  int32_t* positions;
  uint64_t table_stride, page_stride, head_stride, slot_stride;
  uint32_t n_pages, page_shift, kv_heads, head_dim, n_seqs, seq_pages, capacity;
};

// Values at any address that their type allows: the memory unit takes 16 bytes from any 4-byte boundary as it does from a 16-byte one, 4 and
// 8 from any 2-byte one.
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef int32_t i32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
typedef uint16_t u16x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32_any __attribute__((aligned(1)));
typedef __attribute__((address_space(4))) const int32_t constant_i32;   // not written while a kernel runs: read through the scalar cache

inline int refuse(int code, const std::string& what) {
  set_error(what);
  return code;
}

inline bool aligned_to(const void* p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

inline int view_cache(const std::string& who, const tq_cache* c, CacheView* view) {
  if (!c) return refuse(TQ_E_INVALID_ARG, who + ": null cache");
  if (!c->k || !c->v || !c->tables) return refuse(TQ_E_INVALID_ARG, who + ": the cache needs k, v and tables");
  if (c->type != TQ_BF16 && c->type != TQ_INT8) return refuse(TQ_E_UNSUPPORTED, who + ": a cache is TQ_BF16 or TQ_INT8");
  if (c->type == TQ_INT8 && (!c->k_scale || !c->v_scale)) return refuse(TQ_E_INVALID_ARG, who + ": a TQ_INT8 cache needs k_scale and v_scale");
  if (c->page_size < 16 || c->page_size > 1024 || (c->page_size & (c->page_size - 1)))
    return refuse(TQ_E_UNSUPPORTED, who + ": page_size must be a power of two in 16..1024");
  if (c->head_dim == 0 || c->head_dim > 256 || c->head_dim % 16)
    return refuse(TQ_E_UNSUPPORTED, who + ": head_dim must be a multiple of 16 up to 256");
  if (c->kv_heads == 0 || c->kv_heads > 65535 || c->n_pages == 0 || c->n_pages > 0x7FFFFFFFu || c->n_seqs == 0 || c->n_seqs > 65535 || c->seq_pages == 0)
    return refuse(TQ_E_INVALID_ARG, who + ": kv_heads and n_seqs must be in 1..65535, n_pages and seq_pages at least 1");
  const uint64_t capacity = (uint64_t)c->seq_pages * c->page_size;
  if (capacity > (1u << 30)) return refuse(TQ_E_UNSUPPORTED, who + ": more than 2^30 tokens per sequence");
  const uint32_t size = c->type == TQ_BF16 ? 2 : 1;
  const bool whole = !c->page_stride && !c->head_stride && !c->slot_stride;
  if (!whole && (!c->page_stride || !c->head_stride || !c->slot_stride))
    return refuse(TQ_E_INVALID_ARG, who + ": page_stride, head_stride and slot_stride are given together");
  const uint64_t slot = whole ? c->head_dim : c->slot_stride, head = whole ? slot * c->page_size : c->head_stride,
                 page = whole ? head * c->kv_heads : c->page_stride;
  if ((slot * size) % 16 || (head * size) % 16 || (page * size) % 16 || !aligned_to(c->k, 16) || !aligned_to(c->v, 16) ||
      !aligned_to(c->k_scale, 16) || !aligned_to(c->v_scale, 16))
    return refuse(TQ_E_INVALID_ARG, who + ": k, v, their scales and strides must be multiples of 16 bytes");
  if (slot < c->head_dim || (c->kv_heads > 1 && head < c->head_dim) || (c->n_pages > 1 && page < c->head_dim))
    return refuse(TQ_E_INVALID_ARG, who + ": a stride of the cache is smaller than head_dim");
  if (slot * size > (1u << 26)) return refuse(TQ_E_UNSUPPORTED, who + ": slot_stride is more than 2^26 bytes");   // (16 slots are within 32 bits)
  if (!aligned_to(c->tables, 4) || !aligned_to(c->scores, 4) || !aligned_to(c->positions, 4))
    return refuse(TQ_E_INVALID_ARG, who + ": tables, scores and positions must be 4-byte aligned");
  const uint64_t table = c->table_stride ? c->table_stride : c->seq_pages;
  if (table < c->seq_pages) return refuse(TQ_E_INVALID_ARG, who + ": table_stride is smaller than seq_pages");
  *view = CacheView{(char*)c->k, (char*)c->v, c->k_scale, c->v_scale, c->tables, c->scores, c->positions, table, page, head, slot,
                    c->n_pages, (uint32_t)__builtin_ctz(c->page_size), c->kv_heads, c->head_dim, c->n_seqs, c->seq_pages, (uint32_t)capacity};
  return TQ_OK;
}

// The outcome of the launches just made.
inline int launched(const char* who) {
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return TQ_OK;
  return refuse(TQ_E_HIP, std::string(who) + " launch: " + hipGetErrorString(e));
}

// Runs the body of an entry point; no C++ exception leaves the library.
template <typename F>
int contained(const char* who, F&& body) {
  auto say = [&](const char* what) {
    try {
      set_error(std::string(who) + what);
    } catch (...) {   // (no memory for the message either)
    }
  };
  try {
    return body();
  } catch (const std::bad_alloc&) {
    say(": out of host memory");
    return TQ_E_OOM;
  } catch (...) {
    say(": unexpected internal error");
    return TQ_E_HIP;
  }
}

// Maximum and sum over aligned groups of N lanes (N a power of two), the same value in every lane of a group.
template <int N>
__device__ __forceinline__ float group_max(float v) {
#pragma unroll
  for (int d = 1; d < N; d *= 2) v = fmaxf(v, __shfl_xor(v, d));
  return v;
}
template <int N>
__device__ __forceinline__ float group_sum(float v) {
#pragma unroll
  for (int d = 1; d < N; d *= 2) v += __shfl_xor(v, d);
  return v;
}

// Sums over a wavefront's lanes up to and with each.
__device__ __forceinline__ uint32_t wave_prefix_sum(uint32_t v) {
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xf, 0xf, true);
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xf, 0xf, true);
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xf, 0xf, true);
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xf, 0xf, true);
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xa, 0xf, false);   // lane 15 of a row to the next one
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xc, 0xf, false);   // lane 31 to the upper half
  return v;
}

// fmaxf passes over a NaN; this keeps it.
__device__ __forceinline__ float max_or_nan(float a, float b) { return (a != a || b != b) ? __builtin_nanf("") : fmaxf(a, b); }

// The 8-bit quantizer of the weights (tq_encode): round half to even, symmetric; nothing is divided by a scale of zero.
// A row that is not finite has no scale: it reads back as NaN.
__device__ __forceinline__ float scale_of(float absmax) { return absmax < INFINITY ? absmax / 127.f : __builtin_nanf(""); }
__device__ __forceinline__ int quantized(float x, float scale) {
  const float t = rintf(x / scale);
  return scale > 0.f ? (int)fminf(127.f, fmaxf(-127.f, t)) : 0;
}

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b});
}

__device__ __forceinline__ float bf16_value(uint32_t bits) { return __uint_as_float(bits << 16); }

}  // namespace tq
