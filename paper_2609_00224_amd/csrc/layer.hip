// Row operators of a decoder layer: the root-mean-square norm with the
// residual's addition, and the gated activation.
#include <algorithm>
#include <type_traits>

#include "rows.h"

namespace qtea_serve {
namespace {

constexpr int kThreads = 256;
constexpr int64_t kMaxBlocks = 1 << 20;  // of a launch; more rows go round

// Where an operator's result goes: dense, or E4M3 codes and scales.
struct Out {
  char* p;
  uint8_t* scale;
  int64_t stride, scale_stride;  // bytes
  int32_t type;
  bool wide;
};

// The `n` values at element `at` of row r (of `run` values of a token).
__device__ __forceinline__ void store_out(const Out& o, int64_t token, int64_t at, int n, float (&x)[8]) {
  char* row = o.p + token * o.stride;
  const bool wide = o.wide && n == 8;
  if (o.type == QTEA_E4M3) {  // (a block's quad of lanes is here together, n is 8)
    const uint32_t e = block_exponent<QTEA_KV_E4M3>(quad_max(max_bits(x)));
    *reinterpret_cast<u32x2*>(row + at) = block_codes<QTEA_KV_E4M3>(x, e);
    if ((at & 31) == 0) o.scale[token * o.scale_stride + (at >> 5)] = uint8_t(e);
  } else if (o.type == QTEA_F16) {
    store_some<QTEA_F16>(row + 2 * at, n, wide, x);
  } else if (o.type == QTEA_BF16) {
    store_some<QTEA_BF16>(row + 2 * at, n, wide, x);
  } else {
    store_some<QTEA_F32>(row + 4 * at, n, wide, x);
  }
}

__device__ __forceinline__ void load_any(int type, const char* p, int64_t at, int n, bool wide, float (&x)[8]) {
  wide = wide && n == 8;
  if (type == QTEA_F16) load_some<QTEA_F16>(p + 2 * at, n, wide, x);
  else if (type == QTEA_BF16) load_some<QTEA_BF16>(p + 2 * at, n, wide, x);
  else load_some<QTEA_F32>(p + 4 * at, n, wide, x);
}
__device__ __forceinline__ void store_any(int type, char* p, int64_t at, int n, bool wide, const float (&x)[8]) {
  wide = wide && n == 8;
  if (type == QTEA_F16) store_some<QTEA_F16>(p + 2 * at, n, wide, x);
  else if (type == QTEA_BF16) store_some<QTEA_BF16>(p + 2 * at, n, wide, x);
  else store_some<QTEA_F32>(p + 4 * at, n, wide, x);
}

struct NormArgs {
  const char* x;
  char* residual;
  const char* weight;
  int64_t x_stride, residual_stride;  // bytes
  Out out;
  int64_t rows;  // tokens * heads
  int32_t x_type, residual_type, weight_type, heads, dim;
  bool x_wide, residual_wide, weight_wide;
  float eps;
};

// T threads take a row and hold it, 8 NV values each, between the sum of
// squares and the result: every byte moves once.
template <int T, int NV>
__global__ __launch_bounds__(T < kThreads ? kThreads : T) void rms_norm_kernel(const NormArgs a) {
  constexpr int kBlock = T < kThreads ? kThreads : T, kRows = kBlock / T;
  __shared__ float s_sum[kBlock / 64];
  const int t = threadIdx.x % T;
  const int64_t step = int64_t(gridDim.x) * kRows;
  // (whole workgroups go round together: the barriers below)
  for (int64_t row0 = int64_t(blockIdx.x) * kRows; row0 < a.rows; row0 += step) {
    const int64_t row = row0 + threadIdx.x / T;
    const bool in = row < a.rows;
    const int64_t token = a.heads == 1 ? row : row / a.heads, at0 = a.heads == 1 ? 0 : (row - token * a.heads) * a.dim;
    float x[NV][8];
    float sum = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int at = 8 * (j * T + t), n = in ? min(8, a.dim - at) : 0;
      load_any(a.x_type, a.x + (in ? token : 0) * a.x_stride, at0 + at, n, a.x_wide, x[j]);
      if (a.residual) {
        float y[8];
        char* p = a.residual + (in ? token : 0) * a.residual_stride;
        load_any(a.residual_type, p, at0 + at, n, a.residual_wide, y);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[j][i] += y[i];
        store_any(a.residual_type, p, at0 + at, n, a.residual_wide, x[j]);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += x[j][i] * x[j][i];
    }
#pragma unroll
    for (int d = 1; d < (T < 64 ? T : 64); d *= 2) sum += __shfl_xor(sum, d);
    if constexpr (T > 64) {
      __syncthreads();
      if ((threadIdx.x & 63) == 0) s_sum[threadIdx.x / 64] = sum;
      __syncthreads();
      sum = 0.0f;
#pragma unroll
      for (int i = 0; i < kBlock / 64; ++i) sum += s_sum[i];
    }
    const float by = 1.0f / sqrtf(sum / float(a.dim) + a.eps);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int at = 8 * (j * T + t), n = in ? min(8, a.dim - at) : 0;
      if (n <= 0) continue;
      float w[8];
      if (a.weight) load_any(a.weight_type, a.weight, at, n, a.weight_wide, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[j][i] = a.weight ? x[j][i] * by * w[i] : x[j][i] * by;
      store_out(a.out, token, at0 + at, n, x[j]);
    }
  }
}

struct GateArgs {
  const char* gate;
  const char* up;
  int64_t gate_stride, up_stride;  // bytes
  Out out;
  uint32_t octs, total;  // of a row, of all rows
  int32_t type, dim;
  bool gate_wide, up_wide;
};

__global__ __launch_bounds__(kThreads) void silu_mul_kernel(const GateArgs a) {
  for (uint64_t o = uint64_t(blockIdx.x) * kThreads + threadIdx.x; o < a.total; o += uint64_t(gridDim.x) * kThreads) {
    const uint32_t row = uint32_t(o) / a.octs, at = 8 * (uint32_t(o) - row * a.octs);
    const int n = min(8, a.dim - int(at));
    float g[8], u[8];
    load_any(a.type, a.gate + int64_t(row) * a.gate_stride, at, n, a.gate_wide, g);
    load_any(a.type, a.up + int64_t(row) * a.up_stride, at, n, a.up_wide, u);
#pragma unroll
    for (int i = 0; i < 8; ++i) g[i] = g[i] / (1.0f + expf(-g[i])) * u[i];
    store_out(a.out, row, at, n, g);
  }
}

bool dense_type(int type) { return type >= QTEA_F16 && type <= QTEA_F32; }

// The host's checks of an output of `run` values a token; false if not valid.
bool make_out(void* out, int type, int64_t stride, uint8_t* scale, int64_t scale_stride, int64_t run, int64_t dim, Out* o) {
  if (!out || !stride_ok(stride, run)) return false;
  if (type == QTEA_E4M3) {
    if (dim % 32 != 0 || !rows_aligned16(out, stride, type) || !scale || !stride_ok(scale_stride, run / 32)) return false;
  } else if (!dense_type(type) || scale || !aligned_to_elem(out, type)) {
    return false;
  }
  *o = {static_cast<char*>(out), scale, stride * elem_bytes(type), scale_stride, type, rows_aligned16(out, stride, type) && dim % 8 == 0};
  return true;
}

}  // namespace
}  // namespace qtea_serve

using namespace qtea_serve;

extern "C" {

int qtea_rms_norm(const void* x, int x_type, int64_t x_stride, void* residual, int residual_type, int64_t residual_stride,
                  const void* weight, int weight_type, float eps, void* out, int out_type, int64_t out_stride,
                  uint8_t* out_scale, int64_t scale_stride, int64_t tokens, int heads, int64_t dim, void* stream) {
  if (!x || !dense_type(x_type) || tokens < 0 || tokens > INT32_MAX || heads < 1 || heads > 65535 || dim < 1 || dim > QTEA_NORM_MAX_DIM) return QTEA_ERR_INVALID_ARG;
  const int64_t run = heads * dim;
  if (!stride_ok(x_stride, run) || !aligned_to_elem(x, x_type) || !(eps >= 0x1p-126f && eps <= 0x1.fffffep127f)) return QTEA_ERR_INVALID_ARG;
  if (residual && (!dense_type(residual_type) || !stride_ok(residual_stride, run) || !aligned_to_elem(residual, residual_type))) return QTEA_ERR_INVALID_ARG;
  if (residual && (residual == x || residual == out)) return QTEA_ERR_INVALID_ARG;
  if (weight && (!dense_type(weight_type) || !aligned_to_elem(weight, weight_type) || weight == out)) return QTEA_ERR_INVALID_ARG;
  if (x == out && (x_type != out_type || x_stride != out_stride)) return QTEA_ERR_INVALID_ARG;
  NormArgs a;
  if (!make_out(out, out_type, out_stride, out_scale, scale_stride, run, dim, &a.out)) return QTEA_ERR_INVALID_ARG;
  if (tokens == 0) return QTEA_OK;
  a.x = static_cast<const char*>(x), a.residual = static_cast<char*>(residual), a.weight = static_cast<const char*>(weight);
  a.x_stride = x_stride * elem_bytes(x_type), a.residual_stride = residual ? residual_stride * elem_bytes(residual_type) : 0;
  a.rows = tokens * heads, a.heads = heads, a.dim = int32_t(dim), a.eps = eps;
  a.x_type = x_type, a.residual_type = residual_type, a.weight_type = weight_type;
  a.x_wide = rows_aligned16(x, x_stride, x_type) && dim % 8 == 0;
  a.residual_wide = residual && rows_aligned16(residual, residual_stride, residual_type) && dim % 8 == 0;
  a.weight_wide = weight && aligned16(weight);
  const hipStream_t st = static_cast<hipStream_t>(stream);
  auto launch = [&](auto threads, auto nv) {
    constexpr int T = decltype(threads)::value, NV = decltype(nv)::value, block = T < kThreads ? kThreads : T;
    const int64_t blocks = (a.rows + block / T - 1) / (block / T);
    hipLaunchKernelGGL((rms_norm_kernel<T, NV>), dim3(uint32_t(std::min(blocks, kMaxBlocks))), dim3(block), 0, st, a);
  };
  using std::integral_constant;
  if (dim <= 64) launch(integral_constant<int, 8>(), integral_constant<int, 1>());
  else if (dim <= 128) launch(integral_constant<int, 16>(), integral_constant<int, 1>());
  else if (dim <= 256) launch(integral_constant<int, 32>(), integral_constant<int, 1>());
  else if (dim <= 512) launch(integral_constant<int, 64>(), integral_constant<int, 1>());
  else if (dim <= 1024) launch(integral_constant<int, 64>(), integral_constant<int, 2>());
  else if (dim <= 2048) launch(integral_constant<int, 256>(), integral_constant<int, 1>());
  else if (dim <= 4096) launch(integral_constant<int, 256>(), integral_constant<int, 2>());
  else if (dim <= 8192) launch(integral_constant<int, 256>(), integral_constant<int, 4>());
  else if (dim <= 16384) launch(integral_constant<int, 1024>(), integral_constant<int, 2>());
  else if (dim <= 32768) launch(integral_constant<int, 1024>(), integral_constant<int, 4>());
  else launch(integral_constant<int, 1024>(), integral_constant<int, 8>());
  return hipGetLastError() == hipSuccess ? QTEA_OK : QTEA_ERR_HIP;
}

int qtea_silu_mul(const void* gate, const void* up, int type, int64_t gate_stride, int64_t up_stride, void* out,
                  int out_type, int64_t out_stride, uint8_t* out_scale, int64_t scale_stride, int64_t rows, int64_t dim,
                  void* stream) {
  if (!gate || !up || !dense_type(type) || rows < 0 || rows > INT32_MAX || dim < 1 || dim > INT32_MAX) return QTEA_ERR_INVALID_ARG;
  if (!stride_ok(gate_stride, dim) || !stride_ok(up_stride, dim) || !aligned_to_elem(gate, type) || !aligned_to_elem(up, type)) return QTEA_ERR_INVALID_ARG;
  if (out == gate && (out_type != type || out_stride != gate_stride)) return QTEA_ERR_INVALID_ARG;
  if (out == up && (out_type != type || out_stride != up_stride)) return QTEA_ERR_INVALID_ARG;
  const int64_t octs = (dim + 7) / 8;
  if (rows * octs > INT32_MAX) return QTEA_ERR_INVALID_ARG;
  GateArgs a;
  if (!make_out(out, out_type, out_stride, out_scale, scale_stride, dim, dim, &a.out)) return QTEA_ERR_INVALID_ARG;
  if (rows == 0) return QTEA_OK;
  a.gate = static_cast<const char*>(gate), a.up = static_cast<const char*>(up);
  a.gate_stride = gate_stride * elem_bytes(type), a.up_stride = up_stride * elem_bytes(type);
  a.octs = uint32_t(octs), a.total = uint32_t(rows * octs), a.type = type, a.dim = int32_t(dim);
  a.gate_wide = rows_aligned16(gate, gate_stride, type), a.up_wide = rows_aligned16(up, up_stride, type);
  const int64_t blocks = (rows * octs + kThreads - 1) / kThreads;
  hipLaunchKernelGGL(silu_mul_kernel, dim3(uint32_t(std::min(blocks, kMaxBlocks))), dim3(kThreads), 0, static_cast<hipStream_t>(stream), a);
  return hipGetLastError() == hipSuccess ? QTEA_OK : QTEA_ERR_HIP;
}

}  // extern "C"
