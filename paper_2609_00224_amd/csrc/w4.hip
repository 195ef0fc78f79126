// Products of a few rows with a matrix of 4-bit codes.
//
// W [N][K] is packed in tiles of 16 rows by 128 columns, the left operand of four
// matrix instructions: lane (q, r) = 16 q + r of a wave holds row r, columns
// 32 q .. 32 q + 31, a block, as 16 bytes (code j in half j % 2 of byte j / 2).
//   codes   [ceil(N/16)][ceil(K/128)][64 lanes][16 bytes]
//   scales  [ceil(N/16)][ceil(K/512)][64 lanes][4 bytes], byte i that of tile 4 u + i
// Rows and columns past the matrix are zeros.
#include <algorithm>
#include <type_traits>

#include "rows.h"

namespace qtea_serve {
namespace {

constexpr int kThreads = 256;
constexpr int kTile = 1024;       // bytes of a tile's codes
constexpr int kUnitScales = 256;  // bytes of four tiles' scales

struct Layout {
  int64_t strips, tiles, units, scales_at, bytes;  // of 16 rows; tiles and units of four tiles of a strip
};
bool make_layout(int64_t N, int64_t K, Layout* l) {
  if (N < 1 || K < 1 || N > INT32_MAX || K > (int64_t(1) << 30)) return false;
  l->strips = (N + 15) / 16, l->tiles = (K + 127) / 128, l->units = (l->tiles + 3) / 4;
  l->scales_at = l->strips * l->tiles * kTile;
  l->bytes = l->scales_at + l->strips * l->units * kUnitScales;
  return true;
}

struct PackArgs {
  char* w;
  uint8_t* codes;
  uint8_t* scales;
  int64_t stride;  // bytes
  int64_t tiles, units, total;  // total: strips * units * 256 blocks
  int32_t N, K;
  bool wide;
};

// Block b's tile, lane and place: consecutive threads take a strip's tiles of
// one row in turn, so that a wave reads 64 blocks of few rows.
struct Block {
  int64_t strip, tile;
  int lane;
};
__device__ __forceinline__ Block block_of(const PackArgs& a, int64_t b) {
  const int64_t per = 4 * a.units * 4;  // blocks of a row
  const int64_t row = b / per, at = b - row * per;
  return {row >> 4, at >> 2, int((at & 3) * 16 + (row & 15))};
}

template <int TYPE>
__global__ __launch_bounds__(kThreads) void w4_pack_kernel(const PackArgs a) {
  for (int64_t b = int64_t(blockIdx.x) * kThreads + threadIdx.x; b < a.total; b += int64_t(gridDim.x) * kThreads) {
    const Block k = block_of(a, b);
    const int64_t row = k.strip * 16 + (k.lane & 15), col = k.tile * 128 + (k.lane >> 4) * 32;
    float x[4][8];
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t at = col + 8 * j;
      const int n = row < a.N ? int(min(int64_t(8), max(int64_t(0), a.K - at))) : 0;
      load_some<TYPE>(a.w + row * a.stride + at * elem_bytes(TYPE), n, a.wide && n == 8, x[j]);
      m = max(m, max_bits(x[j]));
    }
    const uint32_t e = block_exponent<QTEA_KV_E2M1>(m);
    if (k.tile < a.tiles) {
      u32x4 v;
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = block_codes<QTEA_KV_E2M1>(x[j], e)[0];
      *reinterpret_cast<u32x4*>(a.codes + (k.strip * a.tiles + k.tile) * kTile + k.lane * 16) = v;
    }
    a.scales[(k.strip * a.units + (k.tile >> 2)) * kUnitScales + k.lane * 4 + (k.tile & 3)] = uint8_t(e);
  }
}

template <int TYPE>
__global__ __launch_bounds__(kThreads) void w4_unpack_kernel(const PackArgs a) {
  for (int64_t b = int64_t(blockIdx.x) * kThreads + threadIdx.x; b < a.total; b += int64_t(gridDim.x) * kThreads) {
    const Block k = block_of(a, b);
    const int64_t row = k.strip * 16 + (k.lane & 15), col = k.tile * 128 + (k.lane >> 4) * 32;
    if (k.tile >= a.tiles || row >= a.N) continue;
    const float s = scale_value(a.scales[(k.strip * a.units + (k.tile >> 2)) * kUnitScales + k.lane * 4 + (k.tile & 3)]);
    const u32x4 v = *reinterpret_cast<const u32x4*>(a.codes + (k.strip * a.tiles + k.tile) * kTile + k.lane * 16);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const f32x2 y[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(v[j], 1.0f, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(v[j], 1.0f, 1),
                          __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(v[j], 1.0f, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(v[j], 1.0f, 3)};
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = y[i / 2][i & 1] * s;
      const int64_t at = col + 8 * j;
      const int n = int(min(int64_t(8), max(int64_t(0), a.K - at)));
      store_some<TYPE>(a.w + row * a.stride + at * elem_bytes(TYPE), n, a.wide && n == 8, x);
    }
  }
}

struct GemmArgs {
  const uint8_t* codes;
  const uint8_t* scales;
  const char* x;
  const uint8_t* x_scale;
  char* y;
  int64_t x_stride, x_scale_stride, y_stride;  // bytes
  int32_t N, K, tiles, units, batch, y_type;
  bool x_wide;
};

// The 16-bit type whose matrix instructions a product runs on.  E4M3 activations
// become bf16 values, exactly: the instruction that takes 8-bit operands with
// their scales drops what lies 2^-16 below the largest of its products (measured).
template <int XT>
using Type = std::conditional_t<XT == QTEA_F16, F16, BF16>;

// A lane's 32 activations of a tile as the matrix instructions' right operand.
struct Acts {
  u32x4 v[4];
};

template <int XT>
__device__ __forceinline__ Acts load_acts(const GemmArgs& a, const char* row, const uint8_t* srow, int tile, int q) {
  Acts r;
  const int k0 = tile * 128 + 32 * q;
  if constexpr (XT == QTEA_E4M3) {  // (K is a multiple of 32)
    const bool in = k0 < a.K;
    const float s = scale_of(in ? srow[k0 / 32] : 127u);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const u32x4 zero = {0, 0, 0, 0};
      const u32x4 c = in ? *reinterpret_cast<const u32x4*>(row + k0 + 16 * i) : zero;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        r.v[2 * i + j / 2][j % 2 * 2] = BF16::e4m3<false>(c[j], s);
        r.v[2 * i + j / 2][j % 2 * 2 + 1] = BF16::e4m3<true>(c[j], s);
      }
    }
  } else {
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      const int k = k0 + 8 * m, n = a.K - k;
      if (a.x_wide && n >= 8) {
        r.v[m] = *reinterpret_cast<const u32x4*>(row + 2 * int64_t(k));
      } else {
        const uint16_t* p = reinterpret_cast<const uint16_t*>(row) + k;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t lo = 2 * i < n ? p[2 * i] : 0u, hi = 2 * i + 1 < n ? p[2 * i + 1] : 0u;
          r.v[m][i] = lo | hi << 16;
        }
      }
    }
  }
  return r;
}

// 16 rows of W times 16 of X over 128 columns; `scale`: the lane's block's.  The
// weights are exact in either type.
template <class T>
__device__ __forceinline__ f32x4 tile_product(u32x4 w, uint32_t scale, const Acts& x, f32x4 c) {
  const float s = scale_of(scale);
#pragma unroll
  for (int m = 0; m < 4; ++m) {
    const u32x4 A = {T::template e2m1<0>(w[m], s), T::template e2m1<1>(w[m], s), T::template e2m1<2>(w[m], s), T::template e2m1<3>(w[m], s)};
    c = T::mfma16(A, x.v[m], c);
  }
  return c;
}

__device__ __forceinline__ void store_y(const GemmArgs& a, int b, int64_t n0, f32x4 c) {
  if (b >= a.batch) return;
  char* row = a.y + b * a.y_stride;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (n0 + i >= a.N) break;
    if (a.y_type == QTEA_F32) store1<QTEA_F32>(row + 4 * (n0 + i), c[i]);
    else if (a.y_type == QTEA_F16) store1<QTEA_F16>(row + 2 * (n0 + i), c[i]);
    else store1<QTEA_BF16>(row + 2 * (n0 + i), c[i]);
  }
}

// A workgroup takes 16 rows of W and 16 of X, its waves the tiles in turn.
template <int XT>
__global__ __launch_bounds__(kThreads) void w4_gemm_kernel(const GemmArgs a) {
  __shared__ f32x4 s_sum[kThreads / 64][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, q = lane >> 4;
  const int64_t strip = blockIdx.x;
  const int b = blockIdx.y * 16 + (lane & 15), bx = min(b, a.batch - 1);
  const char* xrow = a.x + bx * a.x_stride;
  const uint8_t* srow = XT == QTEA_E4M3 ? a.x_scale + bx * a.x_scale_stride : nullptr;
  const uint8_t* codes = a.codes + strip * a.tiles * kTile + lane * 16;
  const uint8_t* scales = a.scales + strip * a.units * kUnitScales + lane * 4;
  f32x4 c = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int t = wave; t < a.tiles; t += kThreads / 64) {
    const u32x4 w = *reinterpret_cast<const u32x4*>(codes + int64_t(t) * kTile);
    const uint32_t s = scales[int64_t(t >> 2) * kUnitScales + (t & 3)];
    c = tile_product<Type<XT>>(w, s, load_acts<XT>(a, xrow, srow, t, q), c);
  }
  s_sum[wave][lane] = c;
  __syncthreads();
  if (wave != 0) return;
#pragma unroll
  for (int i = 1; i < kThreads / 64; ++i) c += s_sum[i][lane];
  store_y(a, b, strip * 16 + 4 * q, c);
}

}  // namespace
}  // namespace qtea_serve

using namespace qtea_serve;

namespace {

bool pack_args(const void* packed, int64_t N, int64_t K, const void* W, int type, int64_t w_stride, Layout* l, PackArgs* a) {
  if (!packed || !W || !aligned16(packed) || type < QTEA_F16 || type > QTEA_F32 || !make_layout(N, K, l)) return false;
  if (!stride_ok(w_stride, K) || !aligned_to_elem(W, type)) return false;
  a->w = static_cast<char*>(const_cast<void*>(W));
  a->codes = static_cast<uint8_t*>(const_cast<void*>(packed)), a->scales = a->codes + l->scales_at;
  a->stride = w_stride * elem_bytes(type), a->tiles = l->tiles, a->units = l->units, a->total = l->strips * l->units * 256;
  a->N = int32_t(N), a->K = int32_t(K), a->wide = rows_aligned16(W, w_stride, type);
  return true;
}

template <class Launch>
void for_type(int type, Launch launch) {
  if (type == QTEA_F16) launch(std::integral_constant<int, QTEA_F16>());
  else if (type == QTEA_BF16) launch(std::integral_constant<int, QTEA_BF16>());
  else launch(std::integral_constant<int, QTEA_F32>());
}

dim3 pack_blocks(int64_t total) { return dim3(uint32_t(std::min<int64_t>((total + kThreads - 1) / kThreads, 1 << 20))); }

}  // namespace

extern "C" {

int qtea_w4_packed_bytes(int64_t N, int64_t K, int64_t* out_bytes) {
  Layout l;
  if (!out_bytes || !make_layout(N, K, &l)) return QTEA_ERR_INVALID_ARG;
  *out_bytes = l.bytes;
  return QTEA_OK;
}

int qtea_w4_pack(const void* W, int type, int64_t w_stride, int64_t N, int64_t K, void* packed, int64_t packed_bytes,
                 void* stream) {
  Layout l;
  PackArgs a;
  if (!pack_args(packed, N, K, W, type, w_stride, &l, &a)) return QTEA_ERR_INVALID_ARG;
  if (packed_bytes < l.bytes) return QTEA_ERR_WORKSPACE;
  for_type(type, [&](auto ty) {
    hipLaunchKernelGGL((w4_pack_kernel<decltype(ty)::value>), pack_blocks(a.total), dim3(kThreads), 0, static_cast<hipStream_t>(stream), a);
  });
  return hipGetLastError() == hipSuccess ? QTEA_OK : QTEA_ERR_HIP;
}

int qtea_w4_unpack(const void* packed, int64_t packed_bytes, int64_t N, int64_t K, void* W, int type, int64_t w_stride,
                   void* stream) {
  Layout l;
  PackArgs a;
  if (!pack_args(packed, N, K, W, type, w_stride, &l, &a)) return QTEA_ERR_INVALID_ARG;
  if (packed_bytes < l.bytes) return QTEA_ERR_WORKSPACE;
  for_type(type, [&](auto ty) {
    hipLaunchKernelGGL((w4_unpack_kernel<decltype(ty)::value>), pack_blocks(a.total), dim3(kThreads), 0, static_cast<hipStream_t>(stream), a);
  });
  return hipGetLastError() == hipSuccess ? QTEA_OK : QTEA_ERR_HIP;
}

int qtea_w4_gemm_lowbatch(const void* packed, int64_t packed_bytes, int64_t N, int64_t K, const void* X, int x_type,
                          int64_t x_stride, const uint8_t* x_scale, int64_t x_scale_stride, int batch, void* Y, int y_type,
                          int64_t y_stride, void* stream) {
  Layout l;
  if (!packed || !X || !Y || !aligned16(packed) || !make_layout(N, K, &l)) return QTEA_ERR_INVALID_ARG;
  if (batch < 1 || batch > QTEA_W4_MAX_BATCH) return QTEA_ERR_BATCH;
  if (y_type < QTEA_F16 || y_type > QTEA_F32 || !aligned_to_elem(Y, y_type) || !stride_ok(y_stride, N) || !stride_ok(x_stride, K)) return QTEA_ERR_INVALID_ARG;
  if (x_type == QTEA_E4M3) {
    if (K % 32 != 0 || !rows_aligned16(X, x_stride, x_type) || !x_scale || !stride_ok(x_scale_stride, K / 32)) return QTEA_ERR_INVALID_ARG;
  } else if ((x_type != QTEA_F16 && x_type != QTEA_BF16) || x_scale || !aligned_to_elem(X, x_type)) {
    return QTEA_ERR_INVALID_ARG;
  }
  if (packed_bytes < l.bytes) return QTEA_ERR_WORKSPACE;
  GemmArgs a;
  a.codes = static_cast<const uint8_t*>(packed), a.scales = a.codes + l.scales_at;
  a.x = static_cast<const char*>(X), a.x_scale = x_scale, a.y = static_cast<char*>(Y);
  a.x_stride = x_stride * elem_bytes(x_type), a.x_scale_stride = x_scale_stride, a.y_stride = y_stride * elem_bytes(y_type);
  a.N = int32_t(N), a.K = int32_t(K), a.tiles = int32_t(l.tiles), a.units = int32_t(l.units), a.batch = batch, a.y_type = y_type;
  a.x_wide = rows_aligned16(X, x_stride, x_type);
  const dim3 grid(uint32_t(l.strips), uint32_t((batch + 15) / 16));
  const hipStream_t st = static_cast<hipStream_t>(stream);
  if (x_type == QTEA_F16) hipLaunchKernelGGL((w4_gemm_kernel<QTEA_F16>), grid, dim3(kThreads), 0, st, a);
  else if (x_type == QTEA_BF16) hipLaunchKernelGGL((w4_gemm_kernel<QTEA_BF16>), grid, dim3(kThreads), 0, st, a);
  else hipLaunchKernelGGL((w4_gemm_kernel<QTEA_E4M3>), grid, dim3(kThreads), 0, st, a);
  return hipGetLastError() == hipSuccess ? QTEA_OK : QTEA_ERR_HIP;
}

}  // extern "C"
