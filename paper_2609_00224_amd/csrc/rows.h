// Dense rows a lane takes 8 values of, and blocks of 32 values that share a
// power of two (kv_cache.hip, layer.hip, w4.hip).  Internal to the library.
#ifndef QTEA_ROWS_H_
#define QTEA_ROWS_H_

#include "qtea_layer.h"
#include "serve_common.h"

namespace qtea_serve {

constexpr int elem_bytes(int type) { return type == QTEA_F32 ? 4 : (type == QTEA_E4M3 ? 1 : 2); }

// 8 values of a dense row, 16-byte aligned.
template <int TYPE>
__device__ __forceinline__ void load8(const char* p, float (&x)[8]) {
  if constexpr (TYPE == QTEA_F32) {
    const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = a[i], x[4 + i] = b[i];
  } else if constexpr (TYPE == QTEA_F16) {
    const half8_t v = *reinterpret_cast<const half8_t*>(p);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = float(v[i]);
  } else {
    const u32x4 v = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[2 * i] = __uint_as_float(v[i] << 16), x[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
  }
}
template <int TYPE>
__device__ __forceinline__ void store8(char* p, const float (&x)[8]) {
  if constexpr (TYPE == QTEA_F32) {
    *reinterpret_cast<f32x4*>(p) = f32x4{x[0], x[1], x[2], x[3]};
    *reinterpret_cast<f32x4*>(p + 16) = f32x4{x[4], x[5], x[6], x[7]};
  } else {
    u32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = TYPE == QTEA_F16 ? F16::pack(x[2 * i], x[2 * i + 1]) : BF16::pack(x[2 * i], x[2 * i + 1]);
    *reinterpret_cast<u32x4*>(p) = v;
  }
}

// 8 values as they are loaded, from a row that is read for the last time.
constexpr int kNone = -1;  // in the place of a type: no such operand
template <int T>
struct Raw {
  u32x4 v[T == QTEA_F32 ? 2 : 1];
};
template <>
struct Raw<kNone> {};

template <int T>
__device__ __forceinline__ Raw<T> load_raw(const char* p) {
  Raw<T> r;
  const u32x4* q = reinterpret_cast<const u32x4*>(p);
  r.v[0] = __builtin_nontemporal_load(q);
  if constexpr (T == QTEA_F32) r.v[1] = __builtin_nontemporal_load(q + 1);
  return r;
}
template <int T>
__device__ __forceinline__ void values(const Raw<T>& r, float (&x)[8]) {
  if constexpr (T == QTEA_F32) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(r.v[i / 4][i & 3]);
  } else if constexpr (T == QTEA_F16) {
    const half8_t h = __builtin_bit_cast(half8_t, r.v[0]);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = float(h[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[2 * i] = __uint_as_float(r.v[0][i] << 16), x[2 * i + 1] = __uint_as_float(r.v[0][i] & 0xffff0000u);
  }
}

// One value, aligned to itself.
template <int TYPE>
__device__ __forceinline__ float load1(const char* p) {
  if constexpr (TYPE == QTEA_F32) return *reinterpret_cast<const float*>(p);
  if constexpr (TYPE == QTEA_F16) return float(*reinterpret_cast<const _Float16*>(p));
  return __uint_as_float(uint32_t(*reinterpret_cast<const uint16_t*>(p)) << 16);
}
template <int TYPE>
__device__ __forceinline__ void store1(char* p, float x) {
  if constexpr (TYPE == QTEA_F32) *reinterpret_cast<float*>(p) = x;
  else if constexpr (TYPE == QTEA_F16) *reinterpret_cast<_Float16*>(p) = _Float16(x);
  else *reinterpret_cast<__bf16*>(p) = __bf16(x);
}

// The first n of 8 values, by their own alignment (`wide`: 16-byte aligned, and
// n is 8); zeros past them.
template <int TYPE>
__device__ __forceinline__ void load_some(const char* p, int n, bool wide, float (&x)[8]) {
  if (wide) {
    load8<TYPE>(p, x);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = i < n ? load1<TYPE>(p + i * elem_bytes(TYPE)) : 0.0f;
  }
}
template <int TYPE>
__device__ __forceinline__ void store_some(char* p, int n, bool wide, const float (&x)[8]) {
  if (wide) {
    store8<TYPE>(p, x);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) store1<TYPE>(p + i * elem_bytes(TYPE), x[i]);
  }
}

__device__ __forceinline__ uint32_t quad_max(uint32_t x) {
  const uint32_t y = max(x, uint32_t(__builtin_amdgcn_update_dpp(0, int(x), 0xB1, 0xf, 0xf, true)));  // 1,0,3,2
  return max(y, uint32_t(__builtin_amdgcn_update_dpp(0, int(y), 0x4E, 0xf, 0xf, true)));              // 2,3,0,1
}

// Bits of the largest magnitude of 8 values.
__device__ __forceinline__ uint32_t max_bits(const float (&x)[8]) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(x[i]) & 0x7fffffffu);
  return m;
}

// Biased exponent of a block's scale: the smallest power of two under which
// its largest magnitude `amax` (bits of an fp32) is at most the format's
// largest code, 1.75 * 2^8 or 1.5 * 2^2; within the range for which every
// code times it is an fp16 value.  Not finite: 255.
template <int FMT>
__device__ __forceinline__ uint32_t block_exponent(uint32_t amax) {
  if (amax >= 0x7f800000u) return 255u;
  constexpr int above = FMT == QTEA_KV_E4M3 ? 8 : 2;
  constexpr uint32_t top = FMT == QTEA_KV_E4M3 ? 0x600000u : 0x400000u;
  constexpr int low = FMT == QTEA_KV_E4M3 ? 127 - 15 : 127 - 23, high = FMT == QTEA_KV_E4M3 ? 127 + 7 : 127 + 13;
  const int e = int(amax >> 23) - above + ((amax & 0x7fffffu) > top ? 1 : 0);
  return uint32_t(min(max(e, low), high));
}

// 8 values of a block of scale byte e as codes (x is used up).
template <int FMT>
__device__ __forceinline__ u32x2 block_codes(float (&x)[8], uint32_t e) {
  const bool nan = e == 255u;
  const float inv = __uint_as_float((254u - (nan ? 127u : e)) << 23);  // exact: a power of two
  constexpr float top = FMT == QTEA_KV_E4M3 ? 448.0f : 6.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = __builtin_amdgcn_fmed3f(x[i] * inv, -top, top);
  u32x2 v = {0u, 0u};
  if constexpr (FMT == QTEA_KV_E4M3) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      int q = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i], x[4 * i + 1], 0, false);
      q = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i + 2], x[4 * i + 3], q, true);
      v[i] = nan ? 0x7f7f7f7fu : uint32_t(q);
    }
  } else {
    uint32_t q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, x[0], x[1], 1.0f, 0);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, x[2], x[3], 1.0f, 1);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, x[4], x[5], 1.0f, 2);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, x[6], x[7], 1.0f, 3);
    v[0] = nan ? 0u : q;
  }
  return v;
}

// Host: whether rows `stride` elements apart from `p` are each 16-byte aligned.
inline bool rows_aligned16(const void* p, int64_t stride, int type) { return aligned16(p) && stride * elem_bytes(type) % 16 == 0; }
inline bool aligned_to_elem(const void* p, int type) { return reinterpret_cast<uintptr_t>(p) % elem_bytes(type) == 0; }
// Host: strides whose byte offsets over the call's rows stay far inside 64 bits
// (QTEA_MAX_STRIDE is more than a card's memory holds).
inline bool stride_ok(int64_t stride, int64_t width, int64_t rows) {
  return stride >= width && stride <= QTEA_MAX_STRIDE && (rows <= 1 || stride <= (int64_t(1) << 60) / rows);
}

}  // namespace qtea_serve

#endif  // QTEA_ROWS_H_
