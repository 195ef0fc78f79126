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
#include <algorithm>
#include <type_traits>

#include "rows.h"

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
  int page, off, pos;
  bool some, bad, bad_len;  // whether it is in a sequence, whether it has no page, and that for its sequence's length
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
  Place p = {0, 0, 0, false, false, false};
  if (before == 0) return p;
  const int s = __builtin_amdgcn_readfirstlane(before - 1);
  const int cap = a.b.max_pages << a.page_shift;
  const Seq q = load_seq(a.b, s, cap);
  if (r < q.first || r >= q.first + q.n) return p;
  p.some = true;
  p.bad = p.bad_len = q.bad;
  if (q.bad) return p;
  const int pos = p.pos = q.len - q.n + (r - q.first);
  if (pos < 0) {
    p.off = -1;
    return p;
  }
  p.page = a.b.page_table[int64_t(s) * a.b.max_pages + (pos >> a.page_shift)];
  p.off = pos & ((1 << a.page_shift) - 1);
  p.bad = p.page < 0 || p.page >= a.n_pages;
  return p;
}

// Writes one lane's 8 channels c * 8 .. of a cached row, the quad's lanes
// together (they hold a block).
template <int FMT>
__device__ __forceinline__ void store_cached(const CacheArgs& a, int kv, int64_t row, int c, float (&x)[8]) {
  uint8_t* codes = kv ? a.codes[1] : a.codes[0];
  if constexpr (FMT == QTEA_KV_F16 || FMT == QTEA_KV_BF16) {
    store8<FMT == QTEA_KV_F16 ? QTEA_F16 : QTEA_BF16>(reinterpret_cast<char*>(codes) + row * (2 * a.dim) + 16 * c, x);
  } else {
    const uint32_t e = block_exponent<FMT>(quad_max(max_bits(x)));
    const u32x2 v = block_codes<FMT>(x, e);
    if constexpr (FMT == QTEA_KV_E4M3) *reinterpret_cast<u32x2*>(codes + row * a.dim + 8 * c) = v;
    else *reinterpret_cast<uint32_t*>(codes + row * (a.dim / 2) + 4 * c) = v[0];
    if ((c & 3) == 0) (kv ? a.scales[1] : a.scales[0])[row * (a.dim / 32) + c / 4] = uint8_t(e);
  }
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
  const int64_t row0 = (int64_t(p.page) * a.heads << a.page_shift) + p.off;  // row of head 0; heads a page apart
  for (int o = lane; o < octs; o += 64) {
    if (o != lane) load8<TYPE>(src + o * (8 * kSize), x);
    const int h = o / per, c = o - h * per;
    // (a quad's lanes are together in or out: heads * dim / 8 is a multiple of 4)
    store_cached<FMT>(a, kv, row0 + (int64_t(h) << a.page_shift), c, x);
  }
}

// Keys and queries turned by their positions on the way.  A wave takes a run of
// one token's tasks, a task as many whole heads as it has room for at 8 channels
// a lane, so that a lane's channels are the same in every task: it keeps their
// sines and cosines, which the wave finds once, an angle a lane, and passes
// round through LDS.  The other half of a pair that is rot_dim / 2 channels away is
// loaded a second time (it is in the L1).
//
// An angle is a product of a position (31 bits) and a frequency (24), in double with
// what its rounding left, less the nearest multiple of pi / 2 in two doubles.  Of
// what is left the sine and cosine by their series, also in double (a wave has one
// or two to find), and rounded once.  What is left is at most pi / 4 while the
// quotient's own rounding is small; that reaches a quarter at the largest angle, 2^51,
// and leaves up to 1.25.
//
// HBM bounds it where there are many tokens (19500 of fp16, 32 query and 16 key and
// value heads of 128 channels, into E4M3: 100 us, 464 MB at 4.6 TB/s; a large copy
// reaches 5.2; into E2M1 99 us; keys and values only 48 and 47), with few the chain from
// the sequence's start to the angle's sine (16 tokens of fp32 4.2 us).
struct RotateArgs {
  CacheArgs c;
  const char* q;
  char* q_out;
  int64_t q_stride, q_out_stride;  // bytes
  const float* freq;
  int32_t q_heads, rot, q_out_type;
  int32_t tasks, parts, per_part;  // tasks of a token, waves that share them, tasks a wave
};

constexpr int64_t kFullWaves = 2048;
constexpr int kMaxAngles = QTEA_KV_MAX_DIM / 2;

__device__ __forceinline__ void turn_of(int pos, float freq, float& cs, float& sn) {
  const double p = double(pos), f = double(freq), angle = p * f, rest = __builtin_fma(p, f, -angle);
  const double n = __builtin_rint(angle * 0x1.45f306dc9c883p-1);  // 2 / pi
  // pi / 2 to 106 bits
  double r = __builtin_fma(n, -0x1.921fb54442d18p+0, angle);
  r = __builtin_fma(n, -0x1.1a62633145c07p-54, r) + rest;
  // r^13 / 13! and r^14 / 14! are below 2^-37 up to pi / 4, below 2^-28 up to 1.25
  const double z = r * r;
  const double ps = __builtin_fma(z, __builtin_fma(z, __builtin_fma(z, __builtin_fma(z, -1.0 / 39916800, 1.0 / 362880), -1.0 / 5040), 1.0 / 120), -1.0 / 6);
  const double pc = __builtin_fma(z, __builtin_fma(z, __builtin_fma(z, __builtin_fma(z, __builtin_fma(z, 1.0 / 479001600, -1.0 / 3628800), 1.0 / 40320), -1.0 / 720), 1.0 / 24), -0.5);
  const float s = float(__builtin_fma(r * z, ps, r)), c = float(__builtin_fma(z, pc, 1.0));
  const int quarter = int(int64_t(n) & 3);
  sn = quarter & 1 ? c : s;
  cs = quarter & 1 ? s : c;
  if (quarter & 2) sn = -sn;
  if (quarter == 1 || quarter == 2) cs = -cs;
}

template <int FMT, int TYPE, bool INTERLEAVED, int AHEAD>
__global__ __launch_bounds__(kThreads) void kv_append_rotated_kernel(const RotateArgs a) {
  __shared__ float s_turn[kThreads / 64][2][kMaxAngles];
  const CacheArgs& ca = a.c;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  constexpr int kSize = TYPE == QTEA_F32 ? 4 : 2;
  const int per = ca.dim / 8, heads = 64 / per;  // lanes of a head, heads of a task
  const int hl = lane / per, c = lane - hl * per;
  const int nq = (a.q_heads + heads - 1) / heads, nkv = (ca.heads + heads - 1) / heads;
  const int half = a.rot / 2, h8 = a.rot / 16;
  const bool turned = 8 * c < a.rot;
  const int other = INTERLEAVED || !turned ? 0 : (c < h8 ? h8 : -h8);  // octs to the pairs' other halves
  const int64_t waves = int64_t(ca.b.n_tokens) * a.parts;
  for (int64_t w0 = int64_t(blockIdx.x) * (kThreads / 64); w0 < waves; w0 += int64_t(gridDim.x) * (kThreads / 64)) {
    const int w = __builtin_amdgcn_readfirstlane(int(w0) + wave);
    const int r = w / a.parts, part = w - r * a.parts;
    if (r >= ca.b.n_tokens) return;
    const int first = part * a.per_part, last = min(first + a.per_part, a.tasks);

    // A task's values and the other halves of their pairs, on their way while the tasks
    // before it are turned and stored.  Every lane loads, whatever is stored (the
    // last head again, or past the wave's tasks the token's first key): a
    // number of loads that does not depend on the call lets the wave wait for the
    // one it needs.
    struct Task {
      int seg, head;  // queries, keys, values
      Raw<TYPE> x, y;
    };
    const char* const rows[3] = {a.q + int64_t(r) * a.q_stride, ca.dense[0] + int64_t(r) * ca.stride[0], ca.dense[1] + int64_t(r) * ca.stride[1]};
    const auto fetch = [&](int t) {
      Task k;
      k.seg = t < nq ? 0 : (t < nq + nkv ? 1 : 2);
      k.head = (t - (k.seg == 0 ? 0 : (k.seg == 1 ? nq : nq + nkv))) * heads + hl;
      const char* row = k.seg == 0 ? rows[0] : (k.seg == 1 ? rows[1] : rows[2]);
      const int at = min(k.head, (k.seg == 0 ? a.q_heads : ca.heads) - 1) * ca.dim + 8 * c;
      const bool in = t < last;
      row = in ? row : rows[1];
      k.x = load_raw<TYPE>(row + (in ? at * kSize : 0));
      if constexpr (!INTERLEAVED) k.y = load_raw<TYPE>(row + (in ? (at + 8 * other) * kSize : 0));
      return k;
    };
    Task task[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) task[i] = fetch(first + i);

    const Place p = place_of(ca, r);
    if (!p.some) continue;
    const bool none = p.bad_len || p.pos < 0;
    float cs[8], sn[8];
    if (!none && first < nq + nkv) {
      for (int i = lane; i < half; i += 64) turn_of(p.pos, a.freq[i], s_turn[wave][0][i], s_turn[wave][1][i]);
      // (a wave's LDS accesses are made in order; only the compiler has to keep it)
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      const int base = INTERLEAVED ? 4 * c : (c < h8 ? 8 * c : 8 * c - half);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int at = turned ? base + (INTERLEAVED ? i / 2 : i) : 0;
        const bool low = INTERLEAVED ? (i & 1) == 0 : c < h8;
        const float s = s_turn[wave][1][at];
        cs[i] = turned ? s_turn[wave][0][at] : 1.0f;
        sn[i] = !turned ? 0.0f : (low ? -s : s);  // (negated for the pairs' first halves)
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
    const int64_t row0 = (int64_t(p.bad ? 0 : p.page) * ca.heads << ca.page_shift) + max(p.off, 0);
    const auto finish = [&](const Task& k) {
      if (hl >= heads || k.head >= (k.seg == 0 ? a.q_heads : ca.heads) || (k.seg != 0 && (none || p.bad))) return;
      float x[8];
      values<TYPE>(k.x, x);
      if (none) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = p.bad_len ? __builtin_nanf("") : 0.0f;
      } else if (k.seg != 2 && turned) {
        float y[8];
        if constexpr (INTERLEAVED) {
#pragma unroll
          for (int i = 0; i < 8; ++i) y[i] = x[i ^ 1];
        } else {
          values<TYPE>(k.y, y);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = x[i] * cs[i] + y[i] * sn[i];
      }
      if (k.seg == 0) {
        char* dst = a.q_out + int64_t(r) * a.q_out_stride;
        const int at = k.head * ca.dim + 8 * c;
        if (a.q_out_type == QTEA_F16) store8<QTEA_F16>(dst + at * 2, x);
        else if (a.q_out_type == QTEA_BF16) store8<QTEA_BF16>(dst + at * 2, x);
        else store8<QTEA_F32>(dst + at * 4, x);
      } else {
        store_cached<FMT>(ca, k.seg - 1, row0 + (int64_t(k.head) << ca.page_shift), c, x);
      }
    };
    for (int t = first; t < last; t += AHEAD) {
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        if (t + i < last) finish(task[i]);
        task[i] = fetch(t + i + AHEAD);
      }
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

int qtea_kv_append_rotated(const qtea_kv_cache* cache, const qtea_kv_batch* batch, const void* q, const void* k, const void* v,
                           int type, int64_t q_stride, int64_t k_stride, int64_t v_stride, int n_q_heads, const float* freq,
                           int rot_dim, int interleaved, void* q_out, int q_out_type, int64_t q_out_stride, void* stream) {
  RotateArgs a;
  if (!cache_args(cache, batch, k, v, type, k_stride, v_stride, &a.c)) return QTEA_ERR_INVALID_ARG;
  if (n_q_heads < 0 || n_q_heads > 65535 || !freq || (reinterpret_cast<uintptr_t>(freq) & 3) != 0) return QTEA_ERR_INVALID_ARG;
  if (rot_dim < 16 || rot_dim > cache->head_dim || rot_dim % 16 != 0 || q_out_type < QTEA_F16 || q_out_type > QTEA_F32) return QTEA_ERR_INVALID_ARG;
  if (n_q_heads > 0) {
    const int64_t width = int64_t(n_q_heads) * cache->head_dim;
    if (!q || !q_out || !stride_ok(q_stride, width, batch->n_tokens) || !stride_ok(q_out_stride, width, batch->n_tokens)) return QTEA_ERR_INVALID_ARG;
    if (!rows_aligned16(q, q_stride, type) || !rows_aligned16(q_out, q_out_stride, q_out_type)) return QTEA_ERR_INVALID_ARG;
    if (q == q_out && (type != q_out_type || q_stride != q_out_stride)) return QTEA_ERR_INVALID_ARG;
  } else {
    q_stride = q_out_stride = 0;
  }
  a.q = static_cast<const char*>(q), a.q_out = static_cast<char*>(q_out);
  a.q_stride = q_stride * elem_bytes(type), a.q_out_stride = q_out_stride * elem_bytes(q_out_type);
  a.freq = freq, a.q_heads = n_q_heads, a.rot = rot_dim, a.q_out_type = q_out_type;
  if (a.c.b.n_tokens == 0) return QTEA_OK;
  const int heads = 64 / (cache->head_dim / 8);
  a.tasks = (n_q_heads + heads - 1) / heads + 2 * ((cache->n_heads + heads - 1) / heads);
  // Tasks a wave: all of a token's, or where that leaves the chip without waves
  // (eight a CU of 256) as few as fill it: 16 tokens of 12 tasks 4.0 us at one,
  // 9.1 at twelve; 19500 tokens 228 us at one, 117 at twelve
  // (before tasks were loaded ahead).
  a.per_part = int32_t(std::min<int64_t>(a.tasks, std::max<int64_t>(1, int64_t(a.tasks) * a.c.b.n_tokens / kFullWaves)));
  a.parts = (a.tasks + a.per_part - 1) / a.per_part;
  const int64_t blocks = std::min<int64_t>((int64_t(a.c.b.n_tokens) * a.parts + kThreads / 64 - 1) / (kThreads / 64), 1 << 20);
  for_kernel(cache->format, type, [&](auto fmt, auto ty) {
    constexpr int F = decltype(fmt)::value, T = decltype(ty)::value;
    // (three tasks on the way where a wave has more than one: 19500 tokens 100.5 us,
    // 104 with two, 117 with none)
    const auto kernel = a.per_part > 1 ? (interleaved ? kv_append_rotated_kernel<F, T, true, 3> : kv_append_rotated_kernel<F, T, false, 3>)
                                       : (interleaved ? kv_append_rotated_kernel<F, T, true, 1> : kv_append_rotated_kernel<F, T, false, 1>);
    hipLaunchKernelGGL(kernel, dim3(uint32_t(blocks)), dim3(kThreads), 0, static_cast<hipStream_t>(stream), a);
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
