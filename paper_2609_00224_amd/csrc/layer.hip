// Row operators of a decoder layer: the root-mean-square norm with the
// residual's addition, and the gated activation.
//
// Both move each byte once and are bound by HBM where there are many rows, by the
// call where there are few, but only if the arithmetic is kept down: 8 values a
// thread, conversions fixed at compile time (a branch on the types at each load:
// 8192 x 5120, bf16 to E4M3, 92 us for 61), one exp2 and one reciprocal an activation
// (a correctly rounded quotient and the library's exp: 4099 x 17408, bf16 to
// E4M3, 78 us for 63).  Inputs are read for the last time here and loaded past
// the caches' order (the norm 61 us without, 56 with: 295 MB at 5.3 TB/s); results are
// stored in it, the next operator reads them.  The activation takes 58 us (359
// MB, 6.2 TB/s), 16 x 4096 fp32 with a residual 3.0, 16 x 14336 2.5 (a call in a graph,
// as all of these).
#include <algorithm>
#include <type_traits>

#include "rows.h"

namespace qtea_serve {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxThreads = 1024;
constexpr int64_t kMaxBlocks = 1 << 20;  // of a launch; more rows go round

// Where an operator's result goes: dense, or E4M3 codes and scales.
struct Out {
  char* p;
  uint8_t* scale;
  int64_t stride, scale_stride;  // bytes
  int32_t type;
  bool wide;  // rows are 16-byte aligned and whole octs
};

// The oct at element `at` of a token (x is used up).
template <int T>
__device__ __forceinline__ void store_oct(const Out& o, int64_t token, int64_t at, float (&x)[8]) {
  char* row = o.p + token * o.stride;
  if constexpr (T == QTEA_E4M3) {  // (a block's quad of lanes is here together)
    const uint32_t e = block_exponent<QTEA_KV_E4M3>(quad_max(max_bits(x)));
    *reinterpret_cast<u32x2*>(row + at) = block_codes<QTEA_KV_E4M3>(x, e);
    if ((at & 31) == 0) o.scale[token * o.scale_stride + (at >> 5)] = uint8_t(e);
  } else {
    store8<T>(row + at * elem_bytes(T), x);
  }
}

// -- 8 values of any row ---------------------------------------------------------
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
__device__ __forceinline__ void store_out(const Out& o, int64_t token, int64_t at, int n, float (&x)[8]) {
  if (o.type == QTEA_E4M3) store_oct<QTEA_E4M3>(o, token, at, x);  // (dim is a multiple of 32: n is 8)
  else store_any(o.type, o.p + token * o.stride, at, n, o.wide, x);
}

// -- the norm -------------------------------------------------------------------------
struct NormArgs {
  const char* x;
  char* residual;
  const char* weight;
  int64_t x_stride, residual_stride;  // bytes
  Out out;
  int64_t rows;  // tokens * heads
  int32_t x_type, residual_type, weight_type, heads, dim;
  bool x_wide, residual_wide, weight_wide;
  float eps, inv_dim;
};

// 1 / sqrt(sum / dim + eps): four half ulps from the sum's own.
__device__ __forceinline__ float norm_factor(const NormArgs& a, float sum) {
  return __builtin_amdgcn_rsqf(__builtin_fmaf(sum, a.inv_dim, a.eps));
}

// The sum over 16 lanes (a row of DPP) or a wave, in every lane.
template <int LANES>
__device__ __forceinline__ float lanes_sum(float x) {
  const auto dpp = [](float v, auto ctrl) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), decltype(ctrl)::value, 0xf, 0xf, true)); };
  x += dpp(x, std::integral_constant<int, 0xB1>());   // quad 1,0,3,2
  x += dpp(x, std::integral_constant<int, 0x4E>());   // quad 2,3,0,1
  x += dpp(x, std::integral_constant<int, 0x141>());  // the other quad of 8 (mirrored)
  x += dpp(x, std::integral_constant<int, 0x140>());  // the other 8 of 16 (mirrored)
  if constexpr (LANES == 64) x += __shfl_xor(x, 16), x += __shfl_xor(x, 32);
  return x;
}

// x * by * weight of the oct at `at`.
__device__ __forceinline__ void scale_oct(const NormArgs& a, int at, float by, float (&x)[8]) {
  if (!a.weight) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] *= by;
    return;
  }
  float w[8];
  if (a.weight_type == QTEA_F32) load8<QTEA_F32>(a.weight + 4 * at, w);
  else if (a.weight_type == QTEA_F16) load8<QTEA_F16>(a.weight + 2 * at, w);
  else load8<QTEA_BF16>(a.weight + 2 * at, w);
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = x[i] * by * w[i];
}

// A workgroup takes a row and holds it, 8 NV values a thread, between the sum of
// squares and the result.  (One barrier, which waits for LDS only: the residual's
// stores go on.)
template <int XT, int RT, int OT, int NV>
__global__ __launch_bounds__(kMaxThreads) void rms_norm_row_kernel(const NormArgs a) {
  __shared__ float s_sum[2][kMaxThreads / 64];
  const int per = blockDim.x, t = threadIdx.x;
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const int64_t token = a.heads == 1 ? row : row / a.heads, at0 = a.heads == 1 ? 0 : (row - token * a.heads) * a.dim;
    const char* px = a.x + token * a.x_stride + at0 * elem_bytes(XT);
    char* pr = RT == kNone ? nullptr : a.residual + token * a.residual_stride + at0 * elem_bytes(RT);
    Raw<XT> rx[NV];
    Raw<RT> rr[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int at = 8 * (j * per + t);
      if (at < a.dim) {
        rx[j] = load_raw<XT>(px + at * elem_bytes(XT));
        if constexpr (RT != kNone) rr[j] = load_raw<RT>(pr + at * elem_bytes(RT));
      }
    }
    float x[NV][8], sum = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int at = 8 * (j * per + t);
      if (at < a.dim) {
        values<XT>(rx[j], x[j]);
        if constexpr (RT != kNone) {
          float y[8];
          values<RT>(rr[j], y);
#pragma unroll
          for (int i = 0; i < 8; ++i) x[j][i] += y[i];
          store8<RT>(pr + at * elem_bytes(RT), x[j]);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += x[j][i] * x[j][i];
      }
    }
    sum = lanes_sum<64>(sum);
    if ((t & 63) == 0) s_sum[turn][t / 64] = sum;
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xc07f);  // LDS only
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    sum = 0.0f;
    for (int i = 0; i < per / 64; ++i) sum += s_sum[turn][i];
    turn ^= 1;  // (the other sums are written before the next barrier, read after it)
    const float by = norm_factor(a, sum);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int at = 8 * (j * per + t);
      if (at < a.dim) {
        scale_oct(a, at, by, x[j]);
        store_oct<OT>(a.out, token, at0 + at, x[j]);
      }
    }
  }
}

// Short rows without a residual (the heads of a projection): LANES lanes a row.
template <int XT, int OT, int LANES>
__global__ __launch_bounds__(kThreads) void rms_norm_short_kernel(const NormArgs a) {
  constexpr int kRows = kThreads / LANES;
  const int at = 8 * (threadIdx.x % LANES);
  for (int64_t row0 = int64_t(blockIdx.x) * kRows; row0 < a.rows; row0 += int64_t(gridDim.x) * kRows) {
    const int64_t row = row0 + threadIdx.x / LANES;
    const bool in = row < a.rows && at < a.dim;
    const int64_t token = a.heads == 1 ? row : row / a.heads, at0 = a.heads == 1 ? 0 : (row - token * a.heads) * a.dim;
    float x[8] = {}, sum = 0.0f;
    if (in) values<XT>(load_raw<XT>(a.x + token * a.x_stride + (at0 + at) * elem_bytes(XT)), x);
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += x[i] * x[i];
    const float by = norm_factor(a, lanes_sum<LANES>(sum));
    if (in) {
      scale_oct(a, at, by, x);
      store_oct<OT>(a.out, token, at0 + at, x);
    }
  }
}

// Any types, lengths and alignments, types by branches.  Rows that are not 16-byte
// aligned are loaded value by value (8192 x 5120 of bf16 with a residual into bf16 206
// us, 68 aligned); aligned ones past 16384 values come here too (2560 x 16392 113 us,
// 2560 x 16384 69), and past 32768, at 64 values a thread of 128 registers, some
// spill (1280 x 32768 81 us, 640 x 65536 110).
template <int NV>
__global__ __launch_bounds__(kMaxThreads) void rms_norm_any_kernel(const NormArgs a) {
  __shared__ float s_sum[kMaxThreads / 64];
  const int per = blockDim.x, t = threadIdx.x;
  // (whole workgroups go round together: the barriers below)
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const int64_t token = row / a.heads, at0 = (row - token * a.heads) * a.dim;
    char* pr = a.residual + token * a.residual_stride;
    float x[NV][8], sum = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int at = 8 * (j * per + t), n = min(8, a.dim - at);
      load_any(a.x_type, a.x + token * a.x_stride, at0 + at, n, a.x_wide, x[j]);
      if (a.residual) {
        float y[8];
        load_any(a.residual_type, pr, at0 + at, n, a.residual_wide, y);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[j][i] += y[i];
        store_any(a.residual_type, pr, at0 + at, n, a.residual_wide, x[j]);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += x[j][i] * x[j][i];
    }
    sum = lanes_sum<64>(sum);
    __syncthreads();
    if ((t & 63) == 0) s_sum[t / 64] = sum;
    __syncthreads();
    sum = 0.0f;
    for (int i = 0; i < per / 64; ++i) sum += s_sum[i];
    const float by = norm_factor(a, sum);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int at = 8 * (j * per + t), n = min(8, a.dim - at);
      if (n <= 0) continue;
      float w[8];
      if (a.weight) load_any(a.weight_type, a.weight, at, n, a.weight_wide, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[j][i] = a.weight ? x[j][i] * by * w[i] : x[j][i] * by;
      store_out(a.out, token, at0 + at, n, x[j]);
    }
  }
}

// -- the gated activation -----------------------------------------------------------------
struct GateArgs {
  const char* gate;
  const char* up;
  int64_t gate_stride, up_stride;  // bytes
  Out out;
  uint32_t octs, total;  // of a row, of all rows
  int32_t type, dim;
  bool gate_wide, up_wide;
};

// g / (1 + exp(-g)) u.  exp(-g) = 2^t, t = -g log2(e): for results of 32 bits with what
// the product's rounding left of t (it moves the power by up to 96 half ulps); the
// others round to 2^-12 or more of themselves.
constexpr float kLog2e = 0x1.715476p+0f, kRest = 0x1.4ae0cp-26f;  // log2(e) = kLog2e + kRest to 48 bits
template <bool FULL>
__device__ __forceinline__ float gated(float g, float u) {
  const float t = -g * kLog2e;
  float e = __builtin_amdgcn_exp2f(t);
  if constexpr (FULL) {
    const float rest = __builtin_fmaf(-g, kLog2e, -t) - g * kRest;
    const float better = __builtin_fmaf(e, rest * 0x1.62e43p-1f, e);  // times 2^rest, rest below 2^-17
    e = __builtin_fabsf(t) < 126.0f ? better : e;
  }
  return g * __builtin_amdgcn_rcpf(1.0f + e) * u;
}

// The same below kLow, where the factor leaves the numbers of 32 bits while a large u
// keeps the result among them (and the reciprocal, which has no denormals, gives 0
// for 1 + e from 2^126 on): 1 + e is e there, g 2^n 2^f with n + f = -t, the power taken
// in two steps with u between them.  A gate below -512 is taken as -512: times the
// largest u that is 2^-601, which is 0 as well.
constexpr float kLow = -80.0f;
__device__ float gated_low(float g, float u) {
  g = fmaxf(g, -512.0f);
  const float n = __builtin_rintf(g * kLog2e), f = __builtin_fmaf(g, kRest, __builtin_fmaf(g, kLog2e, -n));
  const float y = __builtin_amdgcn_ldexpf(g * __builtin_amdgcn_exp2f(f), -60) * u;
  return __builtin_amdgcn_ldexpf(y, int(n) + 60);
}

// 8 of them, into g.  (-infinity stays the formula's NaN.)  Few gates are that low:
// asking costs under 1 % (4099 x 17408 of bf16 into bf16 72.5 us for 71.9), all of them
// taking the branch 4 % (74.6).
template <bool FULL>
__device__ __forceinline__ void gated8(float (&g)[8], const float (&u)[8]) {
  float y[8], least = g[0];
#pragma unroll
  for (int k = 0; k < 8; ++k) y[k] = gated<FULL>(g[k], u[k]), least = fminf(least, g[k]);
  if (least < kLow) {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (g[k] < kLow && g[k] >= -0x1.fffffep127f) y[k] = gated_low(g[k], u[k]);
  }
#pragma unroll
  for (int k = 0; k < 8; ++k) g[k] = y[k];
}

template <int T, int OT, int OCTS>
__global__ __launch_bounds__(kThreads) void silu_mul_kernel(const GateArgs a) {
  for (uint64_t o0 = uint64_t(blockIdx.x) * (kThreads * OCTS) + threadIdx.x; o0 < a.total; o0 += uint64_t(gridDim.x) * (kThreads * OCTS)) {
    Raw<T> rg[OCTS], ru[OCTS];
    uint32_t row[OCTS], at[OCTS];
#pragma unroll
    for (int i = 0; i < OCTS; ++i) {
      const uint32_t o = min(uint32_t(o0) + i * kThreads, a.total - 1);  // (total is below 2^31)
      row[i] = o / a.octs, at[i] = 8 * (o - row[i] * a.octs);
      rg[i] = load_raw<T>(a.gate + int64_t(row[i]) * a.gate_stride + int64_t(at[i]) * elem_bytes(T));
      ru[i] = load_raw<T>(a.up + int64_t(row[i]) * a.up_stride + int64_t(at[i]) * elem_bytes(T));
    }
#pragma unroll
    for (int i = 0; i < OCTS; ++i) {
      if (uint32_t(o0) + i * kThreads >= a.total) break;  // (a block's quad of lanes together)
      float g[8], u[8];
      values<T>(rg[i], g);
      values<T>(ru[i], u);
      gated8<OT == QTEA_F32>(g, u);
      store_oct<OT>(a.out, row[i], at[i], g);
    }
  }
}

// Any types, lengths and alignments, value by value where they are not 16 bytes' (4099 x
// 17408 of bf16 into bf16 165 us, 74 aligned).
__global__ __launch_bounds__(kThreads) void silu_mul_any_kernel(const GateArgs a) {
  for (uint64_t o = uint64_t(blockIdx.x) * kThreads + threadIdx.x; o < a.total; o += uint64_t(gridDim.x) * kThreads) {
    const uint32_t row = uint32_t(o) / a.octs, at = 8 * (uint32_t(o) - row * a.octs);
    const int n = min(8, a.dim - int(at));
    float g[8], u[8];
    load_any(a.type, a.gate + int64_t(row) * a.gate_stride, at, n, a.gate_wide, g);
    load_any(a.type, a.up + int64_t(row) * a.up_stride, at, n, a.up_wide, u);
    // (the aligned kernel's arithmetic for each type of result)
    if (a.out.type == QTEA_F32) gated8<true>(g, u);
    else gated8<false>(g, u);
    store_out(a.out, row, at, n, g);
  }
}

// -- the host ---------------------------------------------------------------------------------
using std::integral_constant;

bool dense_type(int type) { return type >= QTEA_F16 && type <= QTEA_F32; }

// The host's checks of an output of `rows` tokens of `run` values; false if not valid.
bool make_out(void* out, int type, int64_t stride, uint8_t* scale, int64_t scale_stride, int64_t run, int64_t dim, int64_t rows, Out* o) {
  if (!out || !stride_ok(stride, run, rows)) return false;
  if (type == QTEA_E4M3) {
    if (dim % 32 != 0 || !rows_aligned16(out, stride, type) || !scale || !stride_ok(scale_stride, run / 32, rows)) return false;
  } else if (!dense_type(type) || scale || !aligned_to_elem(out, type)) {
    return false;
  }
  *o = {static_cast<char*>(out), scale, stride * elem_bytes(type), scale_stride, type, rows_aligned16(out, stride, type) && dim % 8 == 0};
  return true;
}

// `run` with a dense type, or with any output's.
template <class Run>
void for_dense(int type, Run run) {
  if (type == QTEA_F16) run(integral_constant<int, QTEA_F16>());
  else if (type == QTEA_BF16) run(integral_constant<int, QTEA_BF16>());
  else run(integral_constant<int, QTEA_F32>());
}
template <class Run>
void for_out(int type, Run run) {
  if (type == QTEA_E4M3) run(integral_constant<int, QTEA_E4M3>());
  else for_dense(type, run);
}

dim3 capped(int64_t blocks) { return dim3(uint32_t(std::min(blocks, kMaxBlocks))); }
int threads_for(int64_t dim, int nv) { return int((dim + 512 * nv - 1) / (512 * nv)) * 64; }

template <int NV>
void launch_rows(const NormArgs& a, hipStream_t st) {
  for_dense(a.x_type, [&](auto xt) {
    for_out(a.out.type, [&](auto ot) {
      const auto go = [&](auto rt) {
        hipLaunchKernelGGL((rms_norm_row_kernel<decltype(xt)::value, decltype(rt)::value, decltype(ot)::value, NV>), capped(a.rows), dim3(threads_for(a.dim, NV)), 0, st, a);
      };
      if (a.residual) for_dense(a.residual_type, go);
      else go(integral_constant<int, kNone>());
    });
  });
}
template <int LANES>
void launch_short(const NormArgs& a, hipStream_t st) {
  for_dense(a.x_type, [&](auto xt) {
    for_out(a.out.type, [&](auto ot) {
      hipLaunchKernelGGL((rms_norm_short_kernel<decltype(xt)::value, decltype(ot)::value, LANES>), capped((a.rows + kThreads / LANES - 1) / (kThreads / LANES)), dim3(kThreads), 0, st, a);
    });
  });
}
template <int NV>
void launch_any(const NormArgs& a, hipStream_t st) {
  hipLaunchKernelGGL((rms_norm_any_kernel<NV>), capped(a.rows), dim3(threads_for(a.dim, NV)), 0, st, a);
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
  if (!stride_ok(x_stride, run, tokens) || !aligned_to_elem(x, x_type) || !(eps >= 0x1p-126f && eps <= 0x1.fffffep127f)) return QTEA_ERR_INVALID_ARG;
  if (residual && (!dense_type(residual_type) || !stride_ok(residual_stride, run, tokens) || !aligned_to_elem(residual, residual_type))) return QTEA_ERR_INVALID_ARG;
  if (residual && (residual == x || residual == out)) return QTEA_ERR_INVALID_ARG;
  if (weight && (!dense_type(weight_type) || !aligned_to_elem(weight, weight_type) || weight == out)) return QTEA_ERR_INVALID_ARG;
  if (x == out && (x_type != out_type || x_stride != out_stride)) return QTEA_ERR_INVALID_ARG;
  NormArgs a;
  if (!make_out(out, out_type, out_stride, out_scale, scale_stride, run, dim, tokens, &a.out)) return QTEA_ERR_INVALID_ARG;
  if (tokens == 0) return QTEA_OK;
  a.x = static_cast<const char*>(x), a.residual = static_cast<char*>(residual), a.weight = static_cast<const char*>(weight);
  a.x_stride = x_stride * elem_bytes(x_type), a.residual_stride = residual ? residual_stride * elem_bytes(residual_type) : 0;
  a.rows = tokens * heads, a.heads = heads, a.dim = int32_t(dim), a.eps = eps, a.inv_dim = 1.0f / float(dim);
  a.x_type = x_type, a.residual_type = residual_type, a.weight_type = weight_type;
  a.x_wide = rows_aligned16(x, x_stride, x_type) && dim % 8 == 0;
  a.residual_wide = !residual || (rows_aligned16(residual, residual_stride, residual_type) && dim % 8 == 0);
  a.weight_wide = !weight || (aligned16(weight) && dim % 8 == 0);
  const hipStream_t st = static_cast<hipStream_t>(stream);
  const bool wide = a.x_wide && a.residual_wide && a.weight_wide && a.out.wide;
  // 8 values a thread while a workgroup has threads for the row: 16 x 4096 3.8 us
  // with 512 threads, 4.7 with 256 at 16 values, 6.8 at 32 (the first version, in a
  // trace, where today's takes 3.4).
  if (wide && !residual && dim <= 128) launch_short<16>(a, st);
  else if (wide && !residual && dim <= 512) launch_short<64>(a, st);
  else if (wide && dim <= 8 * kMaxThreads) launch_rows<1>(a, st);
  else if (wide && dim <= 16 * kMaxThreads) launch_rows<2>(a, st);
  else if (dim <= 8 * kMaxThreads) launch_any<1>(a, st);
  else if (dim <= 16 * kMaxThreads) launch_any<2>(a, st);
  else if (dim <= 32 * kMaxThreads) launch_any<4>(a, st);
  else launch_any<8>(a, st);
  return hipGetLastError() == hipSuccess ? QTEA_OK : QTEA_ERR_HIP;
}

int qtea_silu_mul(const void* gate, const void* up, int type, int64_t gate_stride, int64_t up_stride, void* out,
                  int out_type, int64_t out_stride, uint8_t* out_scale, int64_t scale_stride, int64_t rows, int64_t dim,
                  void* stream) {
  if (!gate || !up || !dense_type(type) || rows < 0 || rows > INT32_MAX || dim < 1 || dim > INT32_MAX) return QTEA_ERR_INVALID_ARG;
  if (!stride_ok(gate_stride, dim, rows) || !stride_ok(up_stride, dim, rows) || !aligned_to_elem(gate, type) || !aligned_to_elem(up, type)) return QTEA_ERR_INVALID_ARG;
  if (out == gate && (out_type != type || out_stride != gate_stride)) return QTEA_ERR_INVALID_ARG;
  if (out == up && (out_type != type || out_stride != up_stride)) return QTEA_ERR_INVALID_ARG;
  const int64_t octs = (dim + 7) / 8;
  if (rows * octs > INT32_MAX) return QTEA_ERR_INVALID_ARG;
  GateArgs a;
  if (!make_out(out, out_type, out_stride, out_scale, scale_stride, dim, dim, rows, &a.out)) return QTEA_ERR_INVALID_ARG;
  if (rows == 0) return QTEA_OK;
  a.gate = static_cast<const char*>(gate), a.up = static_cast<const char*>(up);
  a.gate_stride = gate_stride * elem_bytes(type), a.up_stride = up_stride * elem_bytes(type);
  a.octs = uint32_t(octs), a.total = uint32_t(rows * octs), a.type = type, a.dim = int32_t(dim);
  a.gate_wide = rows_aligned16(gate, gate_stride, type), a.up_wide = rows_aligned16(up, up_stride, type);
  const hipStream_t st = static_cast<hipStream_t>(stream);
  if (a.gate_wide && a.up_wide && a.out.wide) {
    // two octs a thread once they fill the chip
    for_dense(type, [&](auto t) {
      for_out(out_type, [&](auto ot) {
        constexpr int T = decltype(t)::value, OT = decltype(ot)::value;
        const int64_t n = a.total;
        if (n < (1 << 20)) hipLaunchKernelGGL((silu_mul_kernel<T, OT, 1>), capped((n + kThreads - 1) / kThreads), dim3(kThreads), 0, st, a);
        else hipLaunchKernelGGL((silu_mul_kernel<T, OT, 2>), capped((n + 2 * kThreads - 1) / (2 * kThreads)), dim3(kThreads), 0, st, a);
      });
    });
  } else {
    hipLaunchKernelGGL(silu_mul_any_kernel, capped((int64_t(a.total) + kThreads - 1) / kThreads), dim3(kThreads), 0, st, a);
  }
  return hipGetLastError() == hipSuccess ? QTEA_OK : QTEA_ERR_HIP;
}

}  // extern "C"
