// The paged cache: writing new tokens' keys and values, quantized on the way,
// and reading them back.  Both move each byte once; HBM bounds them, and at
// a few tokens the launch: 23034 fp16 tokens of 8 x 128 channels into E4M3
// 33 us (143 MB at 4.3 TB/s; a large copy reaches 4.6 to 4.8), 40533 read from
// it into fp16 58 us (252 MB, 4.4 TB/s), 16 tokens 3.6 us.  (Passes over several
// caches in turn; over one alone its codes stay in the Infinity Cache, and the
// same read takes 43.)
//
// A block's scale is a power of two, so the division by it and (within the
// exponents written) every decoded value are exact: the only rounding is the
// code's own, and no other order of the arithmetic gives another code.
//
// A wave takes one row (a token) of K or of V: the row's sequence, position
// and page are the same for its lanes, found by one ballot over 64
// sequences' starts while the row's values are already on their way.  A lane
// holds 8 channels, so a block of 32 channels is a quad of lanes and its
// largest magnitude two DPP steps away.
#include <type_traits>

#include "serve_common.h"

namespace qtea_serve {
namespace {

constexpr int kThreads = 256;

struct CacheArgs {
  uint8_t* codes[2];   // K, V
  uint8_t* scales[2];
  char* dense[2];
  int64_t stride[2];   // bytes between a dense operand's tokens
  Batch b;
  int32_t heads, dim, page_shift, n_pages;
};

// Where row r is cached: its page and offset in it.
struct Place {
  int page, off;
  bool some, bad;  // whether it has a position, and whether that has no page
};

__device__ __forceinline__ Place place_of(const CacheArgs& a, int r) {
  // the last sequence that starts at or before r (starts do not decrease, so
  // it is the number of starts <= r, minus one)
  const int lane = threadIdx.x & 63;
  int before = 0;
  for (int s0 = 0; s0 < a.b.n_seq; s0 += 64) {
    const int s = s0 + lane;
    before += __popcll(__ballot(s < a.b.n_seq && a.b.q_start[min(s, a.b.n_seq - 1)] <= r));
  }
  Place p = {0, 0, false, false};
  if (before == 0) return p;
  const int s = __builtin_amdgcn_readfirstlane(before - 1);
  const int cap = a.b.max_pages << a.page_shift;
  const Seq q = load_seq(a.b, s, cap);
  if (r < q.first || r >= q.first + q.n) return p;
  p.some = true;
  p.bad = q.bad;
  if (q.bad) return p;
  const int pos = q.len - q.n + (r - q.first);
  if (pos < 0) {
    p.off = -1;
    return p;
  }
  p.page = a.b.page_table[int64_t(s) * a.b.max_pages + (pos >> a.page_shift)];
  p.off = pos & ((1 << a.page_shift) - 1);
  p.bad = p.page < 0 || p.page >= a.n_pages;
  return p;
}

// 8 values of a dense row.
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

__device__ __forceinline__ uint32_t quad_max(uint32_t x) {
  const uint32_t y = max(x, uint32_t(__builtin_amdgcn_update_dpp(0, int(x), 0xB1, 0xf, 0xf, true)));  // 1,0,3,2
  return max(y, uint32_t(__builtin_amdgcn_update_dpp(0, int(y), 0x4E, 0xf, 0xf, true)));              // 2,3,0,1
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

template <int FMT, int TYPE>
__global__ __launch_bounds__(kThreads) void kv_append_kernel(const CacheArgs a) {
  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane(int(blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6)));
  const int r = w >> 1, kv = w & 1;
  if (r >= a.b.n_tokens) return;
  constexpr int kSize = TYPE == QTEA_F32 ? 4 : 2;
  const char* src = a.dense[kv] + int64_t(r) * a.stride[kv];
  const int octs = a.heads * (a.dim / 8), per = a.dim / 8;
  float x[8];
  if (lane < octs) load8<TYPE>(src + lane * (8 * kSize), x);
  const Place p = place_of(a, r);
  if (!p.some || p.bad || p.off < 0) return;
  uint8_t* codes = kv ? a.codes[1] : a.codes[0];
  uint8_t* scales = kv ? a.scales[1] : a.scales[0];
  const int64_t row0 = (int64_t(p.page) * a.heads << a.page_shift) + p.off;  // row of head 0; heads a page apart
  for (int o = lane; o < octs; o += 64) {
    if (o != lane) load8<TYPE>(src + o * (8 * kSize), x);
    const int h = o / per, c = o - h * per;
    const int64_t row = row0 + (int64_t(h) << a.page_shift);
    if constexpr (FMT == QTEA_KV_F16 || FMT == QTEA_KV_BF16) {
      store8<FMT == QTEA_KV_F16 ? QTEA_F16 : QTEA_BF16>(reinterpret_cast<char*>(codes) + row * (2 * a.dim) + 16 * c, x);
    } else {
      // (a quad's lanes are together in or out: heads * dim / 8 is a multiple of 4)
      uint32_t m = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(x[i]) & 0x7fffffffu);
      const uint32_t e = block_exponent<FMT>(quad_max(m));
      const bool nan = e == 255u;
      const float inv = __uint_as_float((254u - (nan ? 127u : e)) << 23);  // exact: a power of two
      constexpr float top = FMT == QTEA_KV_E4M3 ? 448.0f : 6.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = __builtin_amdgcn_fmed3f(x[i] * inv, -top, top);
      if constexpr (FMT == QTEA_KV_E4M3) {
        u32x2 v;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          int q = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i], x[4 * i + 1], 0, false);
          q = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i + 2], x[4 * i + 3], q, true);
          v[i] = nan ? 0x7f7f7f7fu : uint32_t(q);
        }
        *reinterpret_cast<u32x2*>(codes + row * a.dim + 8 * c) = v;
      } else {
        uint32_t v = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, x[0], x[1], 1.0f, 0);
        v = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(v, x[2], x[3], 1.0f, 1);
        v = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(v, x[4], x[5], 1.0f, 2);
        v = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(v, x[6], x[7], 1.0f, 3);
        *reinterpret_cast<uint32_t*>(codes + row * (a.dim / 2) + 4 * c) = nan ? 0u : v;
      }
      if ((lane & 3) == 0) scales[row * (a.dim / 32) + c / 4] = uint8_t(e);
    }
  }
}

template <int FMT, int TYPE>
__global__ __launch_bounds__(kThreads) void kv_read_kernel(const CacheArgs a) {
  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane(int(blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6)));
  const int r = w >> 1, kv = w & 1;
  if (r >= a.b.n_tokens) return;
  constexpr int kSize = TYPE == QTEA_F32 ? 4 : 2;
  const Place p = place_of(a, r);
  if (!p.some) return;
  char* dst = a.dense[kv] + int64_t(r) * a.stride[kv];
  const uint8_t* codes = kv ? a.codes[1] : a.codes[0];
  const uint8_t* scales = kv ? a.scales[1] : a.scales[0];
  const int octs = a.heads * (a.dim / 8), per = a.dim / 8;
  const bool none = p.bad || p.off < 0;
  const int64_t row0 = (int64_t(none ? 0 : p.page) * a.heads << a.page_shift) + (none ? 0 : p.off);
  for (int o = lane; o < octs; o += 64) {
    const int h = o / per, c = o - h * per;
    const int64_t row = row0 + (int64_t(h) << a.page_shift);
    float x[8];
    if (none) {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = p.bad ? __builtin_nanf("") : 0.0f;
    } else if constexpr (FMT == QTEA_KV_F16 || FMT == QTEA_KV_BF16) {
      load8<FMT == QTEA_KV_F16 ? QTEA_F16 : QTEA_BF16>(reinterpret_cast<const char*>(codes) + row * (2 * a.dim) + 16 * c, x);
    } else {
      const float s = scale_value(scales[row * (a.dim / 32) + c / 4]);
      if constexpr (FMT == QTEA_KV_E4M3) {
        const u32x2 v = *reinterpret_cast<const u32x2*>(codes + row * a.dim + 8 * c);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(int(v[i]), false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(int(v[i]), true);
          x[4 * i] = lo[0] * s, x[4 * i + 1] = lo[1] * s, x[4 * i + 2] = hi[0] * s, x[4 * i + 3] = hi[1] * s;
        }
      } else {
        const uint32_t v = *reinterpret_cast<const uint32_t*>(codes + row * (a.dim / 2) + 4 * c);
        const f32x2 q[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(v, 1.0f, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(v, 1.0f, 1),
                            __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(v, 1.0f, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(v, 1.0f, 3)};
#pragma unroll
        for (int i = 0; i < 4; ++i) x[2 * i] = q[i][0] * s, x[2 * i + 1] = q[i][1] * s;
      }
    }
    store8<TYPE>(dst + o * (8 * kSize), x);
  }
}

// `run` with the kernel for a format and a type.
template <class Run>
void for_kernel(int format, int type, Run run) {
  auto typed = [&](auto fmt) {
    if (type == QTEA_F16) run(fmt, std::integral_constant<int, QTEA_F16>());
    else if (type == QTEA_BF16) run(fmt, std::integral_constant<int, QTEA_BF16>());
    else run(fmt, std::integral_constant<int, QTEA_F32>());
  };
  if (format == QTEA_KV_F16) typed(std::integral_constant<int, QTEA_KV_F16>());
  else if (format == QTEA_KV_BF16) typed(std::integral_constant<int, QTEA_KV_BF16>());
  else if (format == QTEA_KV_E4M3) typed(std::integral_constant<int, QTEA_KV_E4M3>());
  else typed(std::integral_constant<int, QTEA_KV_E2M1>());
}

// The arguments of either kernel; false if they are not valid.
bool cache_args(const qtea_kv_cache* cache, const qtea_kv_batch* batch, const void* k, const void* v, int type,
                int64_t k_stride, int64_t v_stride, CacheArgs* a) {
  if (!cache_ok(cache) || !batch_ok(batch, cache->page_size) || !k || !v || type < QTEA_F16 || type > QTEA_F32) return false;
  const int64_t width = int64_t(cache->n_heads) * cache->head_dim, size = type == QTEA_F32 ? 4 : 2;
  if (k_stride < width || v_stride < width || k_stride > (INT64_MAX >> 34) || v_stride > (INT64_MAX >> 34)) return false;
  if (!aligned16(k) || !aligned16(v) || k_stride * size % 16 != 0 || v_stride * size % 16 != 0) return false;
  if (batch->n_tokens > (int64_t(INT32_MAX) / 2) - 2) return false;  // (a wave per row and tensor)
  a->codes[0] = static_cast<uint8_t*>(cache->k), a->codes[1] = static_cast<uint8_t*>(cache->v);
  a->scales[0] = cache->k_scale, a->scales[1] = cache->v_scale;
  a->dense[0] = static_cast<char*>(const_cast<void*>(k)), a->dense[1] = static_cast<char*>(const_cast<void*>(v));
  a->stride[0] = k_stride * size, a->stride[1] = v_stride * size;
  a->b = kernel_batch(batch);
  a->heads = cache->n_heads, a->dim = cache->head_dim;
  a->page_shift = log2_of(cache->page_size), a->n_pages = int32_t(cache->n_pages);
  return true;
}

uint32_t row_blocks(int n_tokens) { return uint32_t((2 * int64_t(n_tokens) + kThreads / 64 - 1) / (kThreads / 64)); }

}  // namespace
}  // namespace qtea_serve

using namespace qtea_serve;

extern "C" {

int qtea_kv_append(const qtea_kv_cache* cache, const qtea_kv_batch* batch, const void* k, const void* v, int type,
                   int64_t k_stride, int64_t v_stride, void* stream) {
  CacheArgs a;
  if (!cache_args(cache, batch, k, v, type, k_stride, v_stride, &a)) return QTEA_ERR_INVALID_ARG;
  if (a.b.n_tokens == 0) return QTEA_OK;
  for_kernel(cache->format, type, [&](auto fmt, auto ty) {
    hipLaunchKernelGGL((kv_append_kernel<decltype(fmt)::value, decltype(ty)::value>), dim3(row_blocks(a.b.n_tokens)),
                       dim3(kThreads), 0, static_cast<hipStream_t>(stream), a);
  });
  return hipGetLastError() == hipSuccess ? QTEA_OK : QTEA_ERR_HIP;
}

int qtea_kv_read(const qtea_kv_cache* cache, const qtea_kv_batch* batch, void* k, void* v, int type, int64_t k_stride,
                 int64_t v_stride, void* stream) {
  CacheArgs a;
  if (!cache_args(cache, batch, k, v, type, k_stride, v_stride, &a)) return QTEA_ERR_INVALID_ARG;
  if (a.b.n_tokens == 0) return QTEA_OK;
  for_kernel(cache->format, type, [&](auto fmt, auto ty) {
    hipLaunchKernelGGL((kv_read_kernel<decltype(fmt)::value, decltype(ty)::value>), dim3(row_blocks(a.b.n_tokens)),
                       dim3(kThreads), 0, static_cast<hipStream_t>(stream), a);
  });
  return hipGetLastError() == hipSuccess ? QTEA_OK : QTEA_ERR_HIP;
}

}  // extern "C"
