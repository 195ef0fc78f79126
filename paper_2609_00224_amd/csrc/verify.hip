// Verification of drafted tokens against the target's probabilities.
//
// Only one target row per sequence (and the draft's beside it) has to be
// read whole: the one after the accepted drafts.  Those follow from two
// values per draft, which every workgroup of a sequence looks up for itself.
// The row is split into slices, one per workgroup; each sums its weights,
// the last of the sequence's workgroups to arrive finds the slice that holds
// the drawn position and looks that slice through once more.  The sums are
// whole numbers: neither the split nor the order of arrival changes a token.
// Bound by its chain of dependent reads (starts, token, two probabilities,
// the rows, the slices' sums, one slice again), for batches also by HBM: one
// sequence over 32000 entries 6.3 us, 48 over 128257 16.9 us (35 MB on average,
// 2.1 TB/s: 62 % of the waves' cycles are waits).
#include <algorithm>
#include <type_traits>

#include "serve_common.h"

namespace qtea_serve {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxSlices = 64;      // a wave scans their sums
constexpr int kBlock = 8 * kThreads;  // vocabulary entries of one step; slices are whole blocks
constexpr int kTargetBlocks = 2048; // workgroups that keep HBM busy
// A sequence's record in the workspace: its arrival counter and its slices'
// sums, at one place whatever the call's number of sequences.  (The counter has
// a line of its own: arrivals at one line are served one after another.)
constexpr int64_t kCounterBytes = 128;
constexpr int64_t kSeqBytes = kCounterBytes + kMaxSlices * 16;

struct VerifyArgs {
  const char* target;
  const char* draft;
  int64_t target_stride, draft_stride;  // bytes
  const int32_t* tokens;
  const int32_t* q_start;
  const float* u_accept;
  const float* u_sample;
  int32_t* n_accepted;
  int32_t* out_tokens;
  char* records;  // [n_seq], kSeqBytes apart: the counter, then [kMaxSlices][2] sums of max(P - Q, 0) and of P
  int32_t vocab, n_seq, n_rows, n_drafts, max_draft, slices, slice;
};

template <int TYPE>
__device__ __forceinline__ float prob(const char* row, int64_t v) {
  if constexpr (TYPE == QTEA_F32) return reinterpret_cast<const float*>(row)[v];
  if constexpr (TYPE == QTEA_F16) return float(reinterpret_cast<const _Float16*>(row)[v]);
  return __uint_as_float(uint32_t(reinterpret_cast<const uint16_t*>(row)[v]) << 16);
}

// A probability in whole units of 2^-38, floor(2^38 p) (p limited to [0, 1],
// NaN: 0): its units of 2^-19, and what is left of it (exact) in units of 2^-38.
struct Fixed {
  uint32_t hi, lo;
  __device__ __forceinline__ uint64_t whole() const { return (uint64_t(hi) << 19) + lo; }
};
__device__ __forceinline__ Fixed fixed(float p) {
  const float c = __builtin_amdgcn_fmed3f(p > 0.0f ? p : 0.0f, 0.0f, 1.0f) * 0x1p19f;
  Fixed f;
  f.hi = uint32_t(c);
  f.lo = uint32_t((c - float(f.hi)) * 0x1p19f);
  return f;
}
// max(p - q, 0)
__device__ __forceinline__ uint64_t over(Fixed p, Fixed q) {
  const int64_t d = (int64_t(int32_t(p.hi) - int32_t(q.hi)) << 19) + (int32_t(p.lo) - int32_t(q.lo));
  return d > 0 ? uint64_t(d) : 0;
}

// A random number in units of 2^-24.
__device__ __forceinline__ uint64_t unit24(float u) { return u > 0.0f ? min(uint32_t(fminf(u, 1.0f) * 0x1p24f), 0xffffffu) : 0; }

__device__ __forceinline__ uint64_t load64(const uint64_t* p) {
  return __hip_atomic_load(const_cast<uint64_t*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ uint64_t readlane64(uint64_t x, int lane) {
  return uint64_t(uint32_t(__builtin_amdgcn_readlane(int(uint32_t(x)), lane))) | uint64_t(uint32_t(__builtin_amdgcn_readlane(int(uint32_t(x >> 32)), lane))) << 32;
}
template <int CTRL, int ROWS>
__device__ __forceinline__ uint64_t dpp64(uint64_t x) {
  const uint32_t lo = uint32_t(__builtin_amdgcn_update_dpp(0, int(uint32_t(x)), CTRL, ROWS, 0xf, false));
  const uint32_t hi = uint32_t(__builtin_amdgcn_update_dpp(0, int(uint32_t(x >> 32)), CTRL, ROWS, 0xf, false));
  return uint64_t(hi) << 32 | lo;
}
// Inclusive sum over the wave's lanes.
__device__ __forceinline__ uint64_t wave_scan64(uint64_t x) {
  x += dpp64<0x111, 0xf>(x);  // from 1, 2, 4, 8 lanes below in the row of 16
  x += dpp64<0x112, 0xf>(x);
  x += dpp64<0x114, 0xf>(x);
  x += dpp64<0x118, 0xf>(x);
  x += dpp64<0x142, 0xa>(x);  // a row's last lane to the next row
  x += dpp64<0x143, 0xc>(x);  // lane 31 to the upper half
  return x;
}

template <int TYPE, bool DRAFT>
__global__ __launch_bounds__(kThreads) void verify_kernel(const VerifyArgs a) {
  __shared__ uint64_t s_sum[4][2], s_scan[4], s_w[kBlock];
  __shared__ int s_last, s_token;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int s = blockIdx.x / a.slices, slice = blockIdx.x - s * a.slices;
  const int first = min(max(a.q_start[s], 0), a.n_rows), rows = min(max(a.q_start[s + 1], 0), a.n_rows) - first;
  int32_t* out = a.out_tokens + int64_t(s) * (a.max_draft + 1);
  const uint64_t u_sample = unit24(a.u_sample[s]);
  if (rows <= 0) {
    if (slice == 0) {
      for (int i = tid; i <= a.max_draft; i += kThreads) out[i] = -1;
      if (tid == 0) a.n_accepted[s] = 0;
    }
    return;
  }
  // drafts of the sequences before this one: their rows but one each
  int with = 0;
  for (int s0 = 0; s0 < s; s0 += 64) {
    const int t = s0 + lane;
    bool some = false;
    if (t < s) some = min(max(a.q_start[t + 1], 0), a.n_rows) > min(max(a.q_start[t], 0), a.n_rows);
    with += __popcll(__ballot(some));
  }
  const int base = min(max(a.q_start[0], 0), a.n_rows);  // (rows before the first sequence have no drafts)
  const int d0 = first - base - with, n = min(rows - 1, a.max_draft);
  // the first rejected draft, 64 at a time (every wave finds it)
  int acc = n;
  for (int i0 = 0; i0 < n; i0 += 64) {
    const int i = i0 + lane;
    bool ok = true;
    if (i < n) {
      const int d = d0 + i;
      const bool in = d >= 0 && d < a.n_drafts;
      const int x = in ? a.tokens[d] : -1;
      if (x < 0 || x >= a.vocab) ok = false;
      else {
        const uint64_t P = fixed(prob<TYPE>(a.target + (int64_t(first) + i) * a.target_stride, x)).whole();
        const uint64_t Q = DRAFT ? fixed(prob<TYPE>(a.draft + int64_t(d) * a.draft_stride, x)).whole() : uint64_t(1) << 38;
        ok = unit24(a.u_accept[d]) * Q < P << 24;
      }
    }
    const uint64_t no = __ballot(!ok);
    if (no) {
      acc = i0 + __ffsll(static_cast<unsigned long long>(no)) - 1;
      break;
    }
  }
  acc = __builtin_amdgcn_readfirstlane(acc);
  const bool rejected = acc < n;
  const int dr = d0 + acc;
  const bool has_q = rejected && dr >= 0 && dr < a.n_drafts;
  const char* p_row = a.target + (int64_t(first) + acc) * a.target_stride;
  const char* q_row = has_q && DRAFT ? a.draft + int64_t(dr) * a.draft_stride : nullptr;
  const int x_one = has_q && !DRAFT ? a.tokens[dr] : -1;  // where a deterministic draft had its whole mass
  // W and P of entries v + 256 i (0 past the end), i < 8: every load on its way
  // before the first is used, a wave's lanes on consecutive entries
  auto weights = [&](int v, int end, uint64_t (&w)[8], uint64_t (&p)[8]) {
    float x[8], y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = prob<TYPE>(p_row, min(v + kThreads * i, end - 1));
    if (DRAFT && q_row) {
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = prob<TYPE>(q_row, min(v + kThreads * i, end - 1));
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const bool in = v + kThreads * i < end;
      const Fixed f = fixed(in ? x[i] : 0.0f);
      w[i] = p[i] = f.whole();
      if (DRAFT && q_row) w[i] = over(f, fixed(y[i]));
      if (!DRAFT && v + kThreads * i == x_one) w[i] = 0;  // (P is at most 1)
    }
  };

  const int v0 = slice * a.slice, v1 = min(v0 + a.slice, a.vocab);
  uint64_t sw = 0, sp = 0;
  for (int v = v0; v < v1; v += kBlock) {
    uint64_t w[8], p[8];
    weights(v + tid, v1, w, p);
#pragma unroll
    for (int i = 0; i < 8; ++i) sw += w[i], sp += p[i];
  }
  sw = readlane64(wave_scan64(sw), 63), sp = readlane64(wave_scan64(sp), 63);
  if (lane == 0) s_sum[wave][0] = sw, s_sum[wave][1] = sp;
  __syncthreads();
  char* record = a.records + int64_t(s) * kSeqBytes;
  uint64_t* sums = reinterpret_cast<uint64_t*>(record + kCounterBytes);
  if (tid == 0) {
    const uint64_t tw = s_sum[0][0] + s_sum[1][0] + s_sum[2][0] + s_sum[3][0], tp = s_sum[0][1] + s_sum[1][1] + s_sum[2][1] + s_sum[3][1];
    __hip_atomic_store(sums + 2 * slice, tw, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __hip_atomic_store(sums + 2 * slice + 1, tp, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0);  // the sums are there before their arrival is counted
    asm volatile("" ::: "memory");
    uint32_t* counter = reinterpret_cast<uint32_t*>(record);
    const uint32_t before = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    const bool last = before == uint32_t(a.slices - 1);
    if (last) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    s_last = last;
    s_token = -1;
  }
  __syncthreads();
  if (!s_last) return;

  // the slice with the drawn position
  uint64_t tw = lane < a.slices ? load64(sums + 2 * lane) : 0, tp = lane < a.slices ? load64(sums + 2 * lane + 1) : 0;
  uint64_t cw = wave_scan64(tw), cp = wave_scan64(tp);
  const bool from_p = readlane64(cw, 63) == 0;
  if (from_p) cw = cp, tw = tp;
  const uint64_t total = readlane64(cw, 63);
  if (total != 0) {
    const uint64_t r = __umul64hi(total, u_sample << 40);  // floor(U total / 2^24)
    const int at = __popcll(__ballot(cw <= r));  // (below 64: r < total)
    uint64_t before = readlane64(cw, at) - readlane64(tw, at);
    const int b0 = at * a.slice, b1 = min(b0 + a.slice, a.vocab);
    for (int v = b0; v < b1 && before <= r; v += kBlock) {
      // the block's weights by way of LDS: loaded 256 apart, summed 8 in a row
      uint64_t w[8], p[8];
      weights(v + tid, b1, w, p);
#pragma unroll
      for (int i = 0; i < 8; ++i) s_w[tid + kThreads * i] = from_p ? p[i] : w[i];
      __syncthreads();
      uint64_t sum = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += w[i] = s_w[8 * tid + i];
      const uint64_t incl = wave_scan64(sum);
      if (lane == 63) s_scan[wave] = incl;
      __syncthreads();
      uint64_t base = before;
      for (int i = 0; i < wave; ++i) base += s_scan[i];
      uint64_t c = base + incl - sum;
      if (c <= r && base + incl > r) {  // (one thread: the sums do not decrease)
        int k = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          c += w[i];
          k += c <= r ? 1 : 0;
        }
        s_token = v + 8 * tid + k;
      }
      before += s_scan[0] + s_scan[1] + s_scan[2] + s_scan[3];
      __syncthreads();
    }
  }
  const int token = s_token;
  for (int i = tid; i <= a.max_draft; i += kThreads) out[i] = i < acc ? a.tokens[d0 + i] : (i == acc ? token : -1);
  if (tid == 0) a.n_accepted[s] = acc;
}

}  // namespace
}  // namespace qtea_serve

using namespace qtea_serve;

extern "C" {

int qtea_verify_workspace_bytes(int n_seq, int64_t* out_bytes) {
  if (!out_bytes || n_seq < 1) return QTEA_ERR_INVALID_ARG;
  *out_bytes = int64_t(n_seq) * kSeqBytes;
  return QTEA_OK;
}

int qtea_verify_draft(const void* target, const void* draft, int type, int64_t vocab, int64_t target_stride,
                      int64_t draft_stride, const int32_t* tokens, const int32_t* q_start, const float* u_accept,
                      const float* u_sample, int n_seq, int64_t n_rows, int64_t n_drafts, int max_draft,
                      int32_t* n_accepted, int32_t* out_tokens, void* workspace, int64_t workspace_bytes, void* stream) {
  if (!q_start || !u_sample || !n_accepted || !out_tokens || !workspace) return QTEA_ERR_INVALID_ARG;
  if (type < QTEA_F16 || type > QTEA_F32 || vocab < 1 || vocab > (1 << 24) || n_seq < 1 || max_draft < 0 || max_draft > 1023) return QTEA_ERR_INVALID_ARG;
  if (n_rows < 0 || n_rows > INT32_MAX || n_drafts < 0 || n_drafts > INT32_MAX) return QTEA_ERR_INVALID_ARG;
  if ((n_rows > 0 && !target) || (n_drafts > 0 && (!tokens || !u_accept))) return QTEA_ERR_INVALID_ARG;
  if (target_stride < vocab || target_stride > (INT64_MAX >> 34)) return QTEA_ERR_INVALID_ARG;
  if (draft && (draft_stride < vocab || draft_stride > (INT64_MAX >> 34))) return QTEA_ERR_INVALID_ARG;
  const int64_t size = type == QTEA_F32 ? 4 : 2;
  if ((reinterpret_cast<uintptr_t>(target) | reinterpret_cast<uintptr_t>(draft)) % size != 0) return QTEA_ERR_INVALID_ARG;
  if (!aligned16(workspace)) return QTEA_ERR_INVALID_ARG;
  int64_t need = 0;
  qtea_verify_workspace_bytes(n_seq, &need);
  if (workspace_bytes < need) return QTEA_ERR_WORKSPACE;
  VerifyArgs a;
  a.target = static_cast<const char*>(target), a.draft = static_cast<const char*>(draft);
  a.target_stride = target_stride * size, a.draft_stride = draft_stride * size;
  a.tokens = tokens, a.q_start = q_start, a.u_accept = u_accept, a.u_sample = u_sample;
  a.n_accepted = n_accepted, a.out_tokens = out_tokens;
  a.records = static_cast<char*>(workspace);
  a.vocab = int32_t(vocab), a.n_seq = n_seq, a.n_rows = int32_t(n_rows), a.n_drafts = int32_t(n_drafts), a.max_draft = max_draft;
  // Slices of whole blocks: as many as fill the chip, at most kMaxSlices.
  const int64_t want = std::min<int64_t>(std::max<int64_t>(1, kTargetBlocks / n_seq), kMaxSlices);
  a.slice = int32_t((vocab + want * kBlock - 1) / (want * kBlock) * kBlock);
  a.slices = int32_t((vocab + a.slice - 1) / a.slice);
  if (int64_t(a.slices) * n_seq > INT32_MAX) return QTEA_ERR_INVALID_ARG;
  const dim3 grid(uint32_t(a.slices) * uint32_t(n_seq)), block(kThreads);
  const hipStream_t st = static_cast<hipStream_t>(stream);
  auto launch = [&](auto ty) {
    constexpr int TYPE = decltype(ty)::value;
    if (draft) hipLaunchKernelGGL((verify_kernel<TYPE, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((verify_kernel<TYPE, false>), grid, block, 0, st, a);
  };
  if (type == QTEA_F16) launch(std::integral_constant<int, QTEA_F16>());
  else if (type == QTEA_BF16) launch(std::integral_constant<int, QTEA_BF16>());
  else launch(std::integral_constant<int, QTEA_F32>());
  return hipGetLastError() == hipSuccess ? QTEA_OK : QTEA_ERR_HIP;
}

}  // extern "C"
