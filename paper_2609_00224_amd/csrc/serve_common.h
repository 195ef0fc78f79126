// Pieces shared by the serving kernels (kv_cache.hip, paged_attn.hip,
// verify.hip).  Internal to the library.
#ifndef QTEA_SERVE_COMMON_H_
#define QTEA_SERVE_COMMON_H_

#include "qtea_internal.h"
#include "qtea_serve.h"

namespace qtea_serve {

using qtea_detail::u32x4;
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf8_t __attribute__((ext_vector_type(8)));

constexpr int kWave = 64;

// What a kernel reads of a qtea_kv_batch.
struct Batch {
  const int32_t* q_start;
  const int32_t* kv_len;
  const int32_t* page_table;
  int32_t n_tokens, n_seq, max_pages;
};

// A sequence's rows [first, first + n) of the dense operands and its cached
// length; `bad` when the length is outside the page table.
struct Seq {
  int first, n, len;
  bool bad;
};

__device__ __forceinline__ int clamp_row(int r, int n) { return r < 0 ? 0 : (r > n ? n : r); }

__device__ __forceinline__ Seq load_seq(const Batch& b, int s, int capacity) {
  Seq q;
  q.first = clamp_row(b.q_start[s], b.n_tokens);
  q.n = max(0, clamp_row(b.q_start[s + 1], b.n_tokens) - q.first);
  q.len = b.kv_len[s];
  q.bad = q.len < 0 || q.len > capacity;
  if (q.bad) q.len = 0;
  return q;
}

__device__ __forceinline__ uint32_t pack2(float a, float b, half2_t*) {
  const f32x2 v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, half2_t));
}
__device__ __forceinline__ uint32_t pack2(float a, float b, bf2_t*) {
  const f32x2 v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf2_t));
}

// Per 16-bit type: the matrix instructions' operands and the conversions
// from codes (exact: the cache's values are values of both types).
struct F16 {
  typedef _Float16 elem;
  typedef half2_t pair;
  typedef half8_t oct;
  static constexpr uint32_t kExp = 0x7c00u;  // an exponent of all ones: not finite
  // The weights' power of two: what they lack in range below 1 (fp16 is
  // exact to 2^-14 only) they have above it.
  static constexpr float kLift = 6.0f;
  static __device__ __forceinline__ uint32_t pack(float a, float b) { return pack2(a, b, (half2_t*)nullptr); }
  template <bool HI>
  static __device__ __forceinline__ uint32_t e4m3(uint32_t w, float s) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, s, HI));
  }
  template <int I>
  static __device__ __forceinline__ uint32_t e2m1(uint32_t w, float s) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, I));
  }
  static __device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(oct, a), __builtin_bit_cast(oct, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(oct, a), __builtin_bit_cast(oct, b), c, 0, 0, 0);
  }
};
struct BF16 {
  typedef __bf16 elem;
  typedef bf2_t pair;
  typedef bf8_t oct;
  static constexpr uint32_t kExp = 0x7f80u;
  static constexpr float kLift = 0.0f;
  static __device__ __forceinline__ uint32_t pack(float a, float b) { return pack2(a, b, (bf2_t*)nullptr); }
  template <bool HI>
  static __device__ __forceinline__ uint32_t e4m3(uint32_t w, float s) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, HI));
  }
  template <int I>
  static __device__ __forceinline__ uint32_t e2m1(uint32_t w, float s) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, I));
  }
  static __device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(oct, a), __builtin_bit_cast(oct, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(oct, a), __builtin_bit_cast(oct, b), c, 0, 0, 0);
  }
};

// The factor of a scale byte as the scaled conversions take it: they read its
// exponent (0 there is 2^-127, 255 a NaN).
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }
// The same as a number.
__device__ __forceinline__ float scale_value(uint32_t byte) {
  return __uint_as_float(byte == 255u ? 0x7fc00000u : (byte == 0u ? 0x00400000u : byte << 23));
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// Bytes of one token's codes of one head.
__host__ __device__ __forceinline__ int code_row_bytes(int format, int dim) {
  return format == QTEA_KV_E2M1 ? dim / 2 : (format == QTEA_KV_E4M3 ? dim : 2 * dim);
}

inline bool quantized(int format) { return format == QTEA_KV_E4M3 || format == QTEA_KV_E2M1; }

// The host's checks of a cache and a batch.
inline bool cache_ok(const qtea_kv_cache* c) {
  if (!c || !c->k || !c->v || c->format < QTEA_KV_F16 || c->format > QTEA_KV_E2M1) return false;
  if (c->n_heads < 1 || c->n_heads > 65535 || c->head_dim < 32 || c->head_dim > QTEA_KV_MAX_DIM || c->head_dim % 32 != 0) return false;
  if (c->page_size < 16 || c->page_size > QTEA_KV_MAX_PAGE || (c->page_size & (c->page_size - 1)) != 0) return false;
  if (c->n_pages < 1 || c->n_pages > INT32_MAX) return false;
  if (!aligned16(c->k) || !aligned16(c->v)) return false;
  if (quantized(c->format) && (!c->k_scale || !c->v_scale || !aligned16(c->k_scale) || !aligned16(c->v_scale))) return false;
  return true;
}
inline bool batch_ok(const qtea_kv_batch* b, int page_size) {
  if (!b || !b->q_start || !b->kv_len || !b->page_table) return false;
  if (b->n_seq < 1 || b->max_pages < 1 || b->n_tokens < 0 || b->n_tokens > INT32_MAX) return false;
  return int64_t(b->max_pages) * page_size <= QTEA_KV_MAX_LEN;
}
inline Batch kernel_batch(const qtea_kv_batch* b) {
  return {b->q_start, b->kv_len, b->page_table, int32_t(b->n_tokens), b->n_seq, b->max_pages};
}
inline int log2_of(int pow2) { return __builtin_ctz(unsigned(pow2)); }

}  // namespace qtea_serve

#endif  // QTEA_SERVE_COMMON_H_
