// Causal attention of a batch's newest tokens over the paged cache.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "serve_common.h"

namespace qtea_serve {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kTile = 32;              // tokens of one step of a wave
constexpr int kUnit = kTile * kWaves;  // tokens of one step of a workgroup
constexpr int kWgPerCu = 2;

struct AttnArgs {
  const uint8_t* k;
  const uint8_t* v;
  const uint8_t* ks;
  const uint8_t* vs;
  const uint16_t* q;
  uint16_t* out;
  int64_t q_stride, out_stride;  // elements
  Batch b;
  int32_t heads, group, dim, page_shift, n_pages, window;
  float scale;       // times log2(e)
  uint32_t* counters;
  float* part;       // partial rows
  float* part_ml;    // their maxima and sums
};

// ---------------------------------------------------------------------------
// Few rows: a task is one sequence, one key/value head and up to 16 R rows
// (new tokens x the query heads that share the head).  Its tokens are split
// over the waves of a workgroup, and the tasks' units of 128 tokens, one
// after another, in equal runs over the workgroups.
// ---------------------------------------------------------------------------

// The work of sequence s: `nqt` row tasks per head, each of `cnt` units from
// unit t0 on (the same for all: what its first row sees starts there, what
// the last one sees ends there).
struct SeqWork {
  Seq q;
  int t0, cnt, nqt, units;
};

template <int MT>
__device__ __forceinline__ SeqWork seq_work(const AttnArgs& a, int s) {
  SeqWork w;
  w.q = load_seq(a.b, s, a.b.max_pages << a.page_shift);
  const int first = w.q.len - w.q.n + 1;  // positions the first row's prefix holds
  const int lo = a.window > 0 ? max(0, first - a.window) : 0;
  w.t0 = lo / kUnit;
  w.cnt = max(1, (w.q.len + kUnit - 1) / kUnit - w.t0);
  w.nqt = (w.q.n * a.group + MT - 1) / MT;
  w.units = w.nqt * w.cnt * a.heads;
  return w;
}

// Inclusive sum over the wave's lanes.
__device__ __forceinline__ int wave_scan(int x) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int y = __shfl_up(x, d);
    if (lane >= d) x += y;
  }
  return x;
}

// Units before workgroup w's run, of W units over G workgroups; and the
// workgroup that has unit u.
__device__ __forceinline__ int run_first(int w, int W, int G) { return w * (W / G) + min(w, W % G); }
__device__ __forceinline__ int run_owner(int u, int W, int G) {
  const int q = W / G, r = W % G, big = r * (q + 1);
  return u < big ? u / (q + 1) : r + (u - big) / q;
}

// A lane's registers of one tile: the K codes of its token in both 16-token
// halves, the V codes of its 8 tokens, and their blocks' scales.
template <int DP, int FMT>
struct Tile {
  static constexpr int kSteps = DP / 32;                                    // matrix instructions along the channels
  static constexpr int kShrink = FMT == 0 ? 1 : (FMT == 1 ? 2 : 4);         // 16-bit values to codes
  static constexpr int kKWords = 4 * kSteps / kShrink;                      // words of K per half
  static constexpr int kChunk = kKWords >= 4 ? 8 * kShrink : 16;            // channels of one K load
  static constexpr int kChunks = DP / (4 * kChunk);                         // K loads per half
  static constexpr int kCH = DP / 16;                                       // channels per lane in V
  static constexpr int kVWords = (kCH / 2 + kShrink - 1) / kShrink;         // words of V per token
  uint32_t k[2][kKWords];
  uint32_t v[8][kVWords];
  uint32_t ks[2][kChunks];
  uint32_t vs[8];
};

template <int N>
__device__ __forceinline__ void load_words(const uint8_t* p, uint32_t* w) {
  if constexpr (N % 4 == 0) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const u32x4 x = *reinterpret_cast<const u32x4*>(p + 4 * i);
#pragma unroll
      for (int j = 0; j < 4; ++j) w[i + j] = x[j];
    }
  } else if constexpr (N == 2) {
    const u32x2 x = *reinterpret_cast<const u32x2*>(p);
    w[0] = x[0], w[1] = x[1];
  } else {
    w[0] = *reinterpret_cast<const uint32_t*>(p);
  }
}

// Channels 8 i .. 8 i + 7 of the codes in w, as 16-bit pairs.
template <int FMT, class T>
__device__ __forceinline__ void decode_words(const uint32_t* w, int i, float s, uint32_t (&out)[4]) {
  if constexpr (FMT == 0) {
#pragma unroll
    for (int j = 0; j < 4; ++j) out[j] = w[4 * i + j];
  } else if constexpr (FMT == 1) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      out[2 * j] = T::template e4m3<false>(w[2 * i + j], s);
      out[2 * j + 1] = T::template e4m3<true>(w[2 * i + j], s);
    }
  } else {
    out[0] = T::template e2m1<0>(w[i], s);
    out[1] = T::template e2m1<1>(w[i], s);
    out[2] = T::template e2m1<2>(w[i], s);
    out[3] = T::template e2m1<3>(w[i], s);
  }
}

// A 16-bit channel pair is not finite in either half.
template <class T>
__device__ __forceinline__ uint32_t finite_mask(uint32_t x) {
  const uint32_t lo = (x & T::kExp) == T::kExp ? 0u : 0xffffu;
  const uint32_t hi = ((x >> 16) & T::kExp) == T::kExp ? 0u : 0xffff0000u;
  return lo | hi;
}

// x, opaque: what follows from it is computed where it is used and not kept
// in registers across a loop.
__device__ __forceinline__ int fresh(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// The cached row of a sequence's position, for one head (-1: no such page).
__device__ __forceinline__ int64_t cached_row(const AttnArgs& a, const int32_t* table, int h, int pos) {
  const int page = table[pos >> a.page_shift];
  if (page < 0 || page >= a.n_pages) return -1;
  return ((int64_t(page) * a.heads + h) << a.page_shift) + (pos & ((1 << a.page_shift) - 1));
}

// Channel c of a cached V row if it is not finite and a row sees it, for that
// row's sum (a positive weight does not change it); else 0.
template <int FMT, class T>
__device__ __forceinline__ float not_finite_value(const AttnArgs& a, int64_t row, int c, bool sees) {
  c = min(c, a.dim - 1);  // (sums of channels past the last are not used)
  uint32_t w;
  if constexpr (FMT == 0) w = reinterpret_cast<const uint16_t*>(a.v)[row * a.dim + c];
  else if constexpr (FMT == 1) w = T::template e4m3<false>(a.v[row * a.dim + c], scale_of(a.vs[row * (a.dim / 32) + c / 32]));
  else w = T::template e2m1<0>(a.v[row * (a.dim / 2) + c / 2], scale_of(a.vs[row * (a.dim / 32) + c / 32]));  // (all of a block or none)
  const float v = float(__builtin_bit_cast(typename T::pair, w)[0]);
  return sees && !(fabsf(v) < INFINITY) ? v : 0.0f;
}

constexpr int lds_width(int DP) { return DP < 128 ? DP : 128; }  // channels joined at a time

template <int DP, int FMT, class T, int R>
__global__ __launch_bounds__(kThreads, 2) void attn_rows_kernel(const AttnArgs a) {
  using TL = Tile<DP, FMT>;
  constexpr int MT = 16 * R;
  constexpr int CH = TL::kCH, CW = lds_width(DP), CS = CW + 4;  // (+ 4: rows on other banks)
  __shared__ float s_o[kWaves][16][CS];
  __shared__ float s_m[kWaves][MT], s_l[kWaves][MT];
  __shared__ int s_last;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n16 = lane & 15, g = lane >> 4;
  const int D = a.dim, H = a.heads, G = a.group;
  const int rowb = FMT == 0 ? 2 * D : (FMT == 1 ? D : D / 2), nb = D / 32;
  const int pmask = (1 << a.page_shift) - 1;

  // the call's units, and the sequence where this workgroup's run begins
  // (each wave for itself: no barrier)
  int W = 0;
  for (int s0 = 0; s0 < a.b.n_seq; s0 += 64) {
    const int u = s0 + lane < a.b.n_seq ? seq_work<MT>(a, s0 + lane).units : 0;
    W += __builtin_amdgcn_readlane(wave_scan(u), 63);
  }
  const int NG = min(int(gridDim.x), W);
  // neighbouring runs on one XCD: tasks of one head share its cached bytes
  int wg = blockIdx.x;
  if (gridDim.x % 8 == 0) wg = (wg & 7) * (gridDim.x / 8) + (wg >> 3);
  if (wg >= NG) return;
  const int u0 = run_first(wg, W, NG), u1 = run_first(wg + 1, W, NG);
  int s = 0, base = 0;
  for (int s0 = 0; s0 < a.b.n_seq; s0 += 64) {
    const int u = s0 + lane < a.b.n_seq ? seq_work<MT>(a, s0 + lane).units : 0;
    const int sum = wave_scan(u);
    const int before = __popcll(__ballot(base + sum <= u0));
    if (before < 64) {
      s = s0 + before;
      base += before ? __builtin_amdgcn_readlane(sum, before - 1) : 0;
      break;
    }
    base += __builtin_amdgcn_readlane(sum, 63);
  }

  int u = u0;
  while (u < u1 && s < a.b.n_seq) {
    const SeqWork sw = seq_work<MT>(a, s);
    if (u >= base + sw.units) {  // (a sequence without rows has no units)
      base += sw.units;
      ++s;
      continue;
    }
    const int rel = u - base, task = rel / sw.cnt, ua = rel - task * sw.cnt;
    const int ub = min(sw.cnt, ua + (u1 - u));  // units [ua, ub) of the task
    const int h = task / sw.nqt, r0 = (task - h * sw.nqt) * MT;
    const int rows = sw.q.n * G, nrow = min(MT, rows - r0);
    const int64_t token_row0 = sw.q.first;
    const int pos0 = sw.q.len - sw.q.n;  // position of the sequence's first new token

    // The rows: query values in the matrix operand's layout, and what each sees.
    uint32_t qf[R][TL::kSteps][4];
    int hi[R], lo[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int row = 16 * r + n16;
      const bool ok = row < nrow;
      const int rr = r0 + (ok ? row : 0), i = rr / G, hh = rr - i * G;
      const uint16_t* q = a.q + (token_row0 + i) * a.q_stride + int64_t(h * G + hh) * D;
      hi[r] = ok ? max(0, pos0 + i + 1) : 0;
      lo[r] = a.window > 0 ? max(0, pos0 + i + 1 - a.window) : 0;
#pragma unroll
      for (int j = 0; j < TL::kSteps; ++j) {
        constexpr int per = TL::kChunk / 8;
        const int c = (j / per) * (4 * TL::kChunk) + g * TL::kChunk + (j % per) * 8;
        u32x4 x = {0, 0, 0, 0};
        if (ok && c < D) x = *reinterpret_cast<const u32x4*>(q + c);
#pragma unroll
        for (int e = 0; e < 4; ++e) qf[r][j][e] = x[e];
      }
    }
    const int i_first = r0 / G, i_last = (r0 + nrow - 1) / G;
    const int hi_min = max(0, pos0 + i_first + 1), hi_max = max(0, pos0 + i_last + 1);
    const int lo_min = a.window > 0 ? max(0, pos0 + i_first + 1 - a.window) : 0;
    const int lo_max = a.window > 0 ? max(0, pos0 + i_last + 1 - a.window) : 0;

    f32x4 o[R][CH];
    float m[R], l[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      m[r] = -INFINITY, l[r] = 0.0f;
#pragma unroll
      for (int c = 0; c < CH; ++c) o[r][c] = f32x4{0, 0, 0, 0};
    }
    bool bad = sw.q.bad, odd = false;

    const int tile_a = (sw.t0 + ua) * kWaves, tile_b = min((sw.t0 + ub) * kWaves, (hi_max + kTile - 1) / kTile);
    const int32_t* table = a.b.page_table + int64_t(s) * a.b.max_pages;
    for (int t = tile_a + wave; t < tile_b; t += kWaves) {
      const int tok0 = t * kTile;
      if (tok0 + kTile <= lo_min) continue;
      TL x;
      int64_t prow[2];  // cached row of the halves' first tokens
#pragma unroll
      for (int sub = 0; sub < 2; ++sub) {
        const int tok = min(tok0 + 16 * sub, (hi_max - 1) & ~15);  // (a half past the end repeats the last one)
        int page = table[tok >> a.page_shift];
        if (page < 0 || page >= a.n_pages) {
          // a half below the window holds no visible token: its page may be gone
          bad = bad || tok + 16 > lo_min;
          page = 0;
        }
        prow[sub] = ((int64_t(page) * H + h) << a.page_shift) + (tok & pmask);
      }
#pragma unroll
      for (int sub = 0; sub < 2; ++sub) {
        const uint8_t* kp = a.k + prow[sub] * rowb + n16 * rowb;
        const uint8_t* sp = FMT ? a.ks + prow[sub] * nb + n16 * nb : nullptr;
#pragma unroll
        for (int i = 0; i < TL::kChunks; ++i) {
          const int c = i * (4 * TL::kChunk) + g * TL::kChunk, cc = c < D ? c : 0;
          load_words<TL::kKWords / TL::kChunks>(kp + (FMT == 0 ? 2 * cc : (FMT == 1 ? cc : cc / 2)), x.k[sub] + i * (TL::kKWords / TL::kChunks));
          if constexpr (FMT != 0) x.ks[sub][i] = sp[cc / 32];
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int c = n16 * CH < D ? n16 * CH : 0;
          const uint8_t* vp = a.v + prow[sub] * rowb + (4 * g + j) * rowb + (FMT == 0 ? 2 * c : (FMT == 1 ? c : c / 2));
          if constexpr (FMT == 2 && CH == 4) x.v[4 * sub + j][0] = *reinterpret_cast<const uint16_t*>(vp);
          else load_words<TL::kVWords>(vp, x.v[4 * sub + j]);
          if constexpr (FMT != 0) x.vs[4 * sub + j] = a.vs[prow[sub] * nb + (4 * g + j) * nb + c / 32];
        }
      }
      // scores: K (16 tokens x channels) times the rows' queries
      f32x4 sc[R][2];
#pragma unroll
      for (int sub = 0; sub < 2; ++sub) {
#pragma unroll
        for (int r = 0; r < R; ++r) sc[r][sub] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < TL::kSteps; ++j) {
          constexpr int per = TL::kChunk / 8;
          uint32_t kw[4];
          decode_words<FMT, T>(x.k[sub], j, FMT ? scale_of(x.ks[sub][j / per]) : 1.0f, kw);
#pragma unroll
          for (int r = 0; r < R; ++r)
            sc[r][sub] = T::mfma16(u32x4{kw[0], kw[1], kw[2], kw[3]}, u32x4{qf[r][j][0], qf[r][j][1], qf[r][j][2], qf[r][j][3]}, sc[r][sub]);
        }
      }
      // V: pairs of tokens per channel from pairs of channels per token
      uint32_t vt[8][CH / 2];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float s = FMT ? scale_of(x.vs[j]) : 1.0f;
        if constexpr (CH == 4) {
          if constexpr (FMT == 0) vt[j][0] = x.v[j][0], vt[j][1] = x.v[j][1];
          else if constexpr (FMT == 1) vt[j][0] = T::template e4m3<false>(x.v[j][0], s), vt[j][1] = T::template e4m3<true>(x.v[j][0], s);
          else vt[j][0] = T::template e2m1<0>(x.v[j][0], s), vt[j][1] = T::template e2m1<1>(x.v[j][0], s);
        } else {
#pragma unroll
          for (int i = 0; i < CH / 8; ++i) {
            uint32_t w[4];
            decode_words<FMT, T>(x.v[j], i, s, w);
#pragma unroll
            for (int e = 0; e < 4; ++e) vt[j][4 * i + e] = w[e];
          }
        }
      }
      const bool edge = tok0 + kTile > hi_min || tok0 < lo_max;
      if (edge) {
        // What a row does not see has no weight; and values that are not
        // finite are left out, since 0 times them is not 0: not_finite_value
        // gives them to the rows that see them.
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
          for (int sub = 0; sub < 2; ++sub)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int tok = tok0 + 16 * sub + 4 * g + i;
              if (tok >= hi[r] || tok < lo[r]) sc[r][sub][i] = -INFINITY;
            }
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
          for (int e = 0; e < CH / 2; ++e) {
            const uint32_t fm = finite_mask<T>(vt[j][e]);
            odd |= fm != 0xffffffffu && tok0 + 16 * (j / 4) + 4 * g + j % 4 < hi_max;
            vt[j][e] &= fm;
          }
      }
      // softmax: the running maximum moves only when a score passes it by 8 powers of two
      uint32_t pw[R][4];
#pragma unroll
      for (int r = 0; r < R; ++r) {
        float top = -INFINITY;
#pragma unroll
        for (int sub = 0; sub < 2; ++sub)
#pragma unroll
          for (int i = 0; i < 4; ++i) top = fmaxf(top, sc[r][sub][i]);
        if (__ballot(top * a.scale > m[r] + 8.0f)) {
          top = fmaxf(top, __shfl_xor(top, 16));
          top = fmaxf(top, __shfl_xor(top, 32));
          const float now = fmaxf(m[r], top * a.scale);
          const float f = m[r] == now ? 1.0f : exp2f(m[r] - now);
          m[r] = now;
          l[r] *= f;
#pragma unroll
          for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[r][c][i] *= f;
        }
        const float off = (m[r] == -INFINITY ? 0.0f : -m[r]) + T::kLift;
#pragma unroll
        for (int sub = 0; sub < 2; ++sub)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            sc[r][sub][i] = __builtin_amdgcn_exp2f(fmaf(sc[r][sub][i], a.scale, off));
            l[r] += sc[r][sub][i];
          }
#pragma unroll
        for (int i = 0; i < 4; ++i) pw[r][i] = T::pack(sc[r][i / 2][2 * (i % 2)], sc[r][i / 2][2 * (i % 2) + 1]);
      }
      // V^T (16 of a lane row's channels x 32 tokens) times the weights
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        u32x4 w;
#pragma unroll
        for (int jj = 0; jj < 4; ++jj)
          w[jj] = __builtin_amdgcn_perm(vt[2 * jj + 1][c / 2], vt[2 * jj][c / 2], c % 2 ? 0x07060302u : 0x05040100u);
#pragma unroll
        for (int r = 0; r < R; ++r) o[r][c] = T::mfma16(w, u32x4{pw[r][0], pw[r][1], pw[r][2], pw[r][3]}, o[r][c]);
      }
    }
    if (__builtin_expect(__ballot(odd) != 0, 0)) {
      for (int t = tile_a + wave; t < tile_b; t += kWaves) {
        const int tok0 = t * kTile;
        if (!(tok0 + kTile > hi_min || tok0 < lo_max)) continue;
        for (int tok = max(tok0, lo_min); tok < min(tok0 + kTile, hi_max); ++tok) {
          const int64_t row = cached_row(a, table, h, tok);
          if (row < 0) continue;
          const int c0 = fresh(4 * g * CH);
#pragma unroll
          for (int r = 0; r < R; ++r) {
            const bool sees = tok < hi[r] && tok >= lo[r];
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
              for (int e = 0; e < 4; ++e) o[r][c][e] += not_finite_value<FMT, T>(a, row, c0 + e * CH + c, sees);
          }
        }
      }
    }
    // this lane's tokens of the sums: over the four lanes of a row
#pragma unroll
    for (int r = 0; r < R; ++r) {
      l[r] += __shfl_xor(l[r], 16);
      l[r] += __shfl_xor(l[r], 32);
      if (bad) l[r] = __builtin_nanf("");
      if (g == 0) s_m[wave][16 * r + n16] = m[r], s_l[wave][16 * r + n16] = l[r];
    }
    __syncthreads();

    // The waves' rows joined: each at the common maximum, summed in wave order.
    const bool whole = ua == 0 && ub == sw.cnt;
    const int slot = 2 * wg + (ua == 0 ? 1 : 0);
    float* part = a.part + int64_t(slot) * (MT * DP);
    float* part_ml = a.part_ml + int64_t(slot) * (2 * MT);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int row = 16 * r + n16;
      float M = s_m[0][row];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) M = fmaxf(M, s_m[w][row]);
      const float f = m[r] == M ? 1.0f : exp2f(m[r] - M);
#pragma unroll
      for (int half = 0; half < DP / CW; ++half) {
        if (DP == CW || (4 * g * CH) / CW == half) {
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int c = 0; c < CH; ++c) s_o[wave][n16][(4 * g + i) * CH + c - half * CW] = o[r][c][i] * f;
        }
        __syncthreads();
        for (int e = tid; e < 16 * (CW / 4); e += kThreads) {
          const int rw = e / (CW / 4), c4 = (e % (CW / 4)) * 4, row2 = 16 * r + rw, ch = half * CW + c4;
          float M2 = s_m[0][row2];
#pragma unroll
          for (int w = 1; w < kWaves; ++w) M2 = fmaxf(M2, s_m[w][row2]);
          float L = 0;
          f32x4 acc = {0, 0, 0, 0};
#pragma unroll
          for (int w = 0; w < kWaves; ++w) {
            const float mw = s_m[w][row2];
            L += s_l[w][row2] * (mw == M2 ? 1.0f : exp2f(mw - M2));
            acc += *reinterpret_cast<const f32x4*>(&s_o[w][rw][c4]);
          }
          if (row2 < nrow && ch < D) {
            if (whole) {
              const int rr = r0 + row2, i = rr / G, hh = rr - i * G;
              // (no position: nothing was summed)
              const float inv = pos0 + i < 0 && L == 0.0f ? 0.0f : 1.0f / L;
              uint32_t w2[2] = {T::pack(acc[0] * inv, acc[1] * inv), T::pack(acc[2] * inv, acc[3] * inv)};
              uint16_t* dst = a.out + (token_row0 + i) * a.out_stride + int64_t(h * G + hh) * D + ch;
              *reinterpret_cast<u32x2*>(dst) = u32x2{w2[0], w2[1]};
            } else {
#pragma unroll
              for (int i = 0; i < 4; ++i) qtea_detail::store_coherent(part + row2 * DP + ch + i, acc[i]);
              if (ch == 0) {
                qtea_detail::store_coherent(part_ml + row2, M2);
                qtea_detail::store_coherent(part_ml + MT + row2, L);
              }
            }
          }
        }
        __syncthreads();
      }
    }
    if (!whole) {
      // The last of the task's workgroups to arrive sums their parts, in run order.
      const int first_u = u - ua, ga = run_owner(first_u, W, NG), gb = run_owner(first_u + sw.cnt - 1, W, NG);
      __builtin_amdgcn_s_waitcnt(0);  // the part is complete before its arrival is counted
      __syncthreads();
      if (tid == 0) {
        const uint32_t before = __hip_atomic_fetch_add(a.counters + ga, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        const bool last = before == uint32_t(gb - ga);
        if (last) __hip_atomic_store(a.counters + ga, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        s_last = last;
      }
      __syncthreads();
      if (s_last) {
        for (int e = tid; e < nrow * (DP / 4); e += kThreads) {
          const int row2 = e / (DP / 4), ch = (e % (DP / 4)) * 4;
          if (ch >= D) continue;
          float M2 = -INFINITY, L = 0;
          f32x4 acc = {0, 0, 0, 0};
          for (int w = ga; w <= gb; ++w) {
            const int64_t sl = 2 * w + (w == ga ? 1 : 0);
            const float mw = qtea_detail::load_coherent(a.part_ml + sl * (2 * MT) + row2);
            const float lw = qtea_detail::load_coherent(a.part_ml + sl * (2 * MT) + MT + row2);
            f32x4 ow;
#pragma unroll
            for (int i = 0; i < 4; ++i) ow[i] = qtea_detail::load_coherent(a.part + sl * (MT * DP) + row2 * DP + ch + i);
            const float now = fmaxf(M2, mw);
            const float fa = M2 == now ? 1.0f : exp2f(M2 - now), fb = mw == now ? 1.0f : exp2f(mw - now);
            M2 = now;
            L = L * fa + lw * fb;
            acc = acc * fa + ow * fb;
          }
          const int rr = r0 + row2, i = rr / G, hh = rr - i * G;
          const float inv = pos0 + i < 0 && L == 0.0f ? 0.0f : 1.0f / L;
          uint16_t* dst = a.out + (token_row0 + i) * a.out_stride + int64_t(h * G + hh) * D + ch;
          *reinterpret_cast<u32x2*>(dst) = u32x2{T::pack(acc[0] * inv, acc[1] * inv), T::pack(acc[2] * inv, acc[3] * inv)};
        }
        __syncthreads();
      }
    }
    u += ub - ua;
  }
}

// ---------------------------------------------------------------------------
// Many rows: a task is one sequence, one key/value head and 128 rows, 32 per
// wave; the workgroup stages tiles of tokens through LDS for its four waves.
// Where there are few tasks their tokens are split into `parts`.
// ---------------------------------------------------------------------------
constexpr int kTaskRows = 128;
constexpr int kMinPart = 4;   // tiles of a part, at least
constexpr int kMaxParts = 16; // of a task

template <int DP, int FMT>
struct Stage {
  static constexpr int kTok = DP <= 128 ? 64 : 32;          // tokens of a tile
  static constexpr int kBlocks = kTok / 32;
  static constexpr int kChunk = FMT == 0 ? 8 : (FMT == 1 ? 16 : 32);  // channels of a 16-byte load
  static constexpr int kPer = DP / kChunk;                   // chunks per token
  static constexpr int kTotal = kTok * kPer;
  static constexpr int kLoads = (kTotal + kThreads - 1) / kThreads;  // per thread, of K and of V
  static constexpr int kBytes = kTok * DP * 2;               // of K (or V) in LDS
};

// Tiles in LDS, rows of DP 16-bit values, arranged so that the lanes of a read
// fall on different banks: K's 16-byte chunks are permuted by the token (read
// as rows of 16 bytes per lane), V's 64-byte granules (read transposed, four
// tokens x 32 channels at a time).
template <int DP>
__device__ __forceinline__ uint32_t k_place(int tok, int chunk) {
  return uint32_t(tok * (2 * DP) + ((chunk ^ (tok & (DP == 64 ? 7 : 15))) << 4));
}
template <int DP>
__device__ __forceinline__ uint32_t v_place(int tok, int chunk) {
  const int f = DP == 64 ? (tok >> 1) & 1 : tok & 3;
  return uint32_t(tok * (2 * DP) + (((chunk >> 2) ^ f) << 6) + ((chunk & 3) << 4));
}

typedef short s16x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ u32x2 lds_read_transposed(const char* p) {
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p));
}

template <int DP, int FMT, class T>
__global__ __launch_bounds__(kThreads, DP == 256 ? 1 : 2) void attn_tile_kernel(const AttnArgs a, int parts) {
  using ST = Stage<DP, FMT>;
  constexpr int KT = ST::kTok, NB = ST::kBlocks, CB = DP / 32, NL = ST::kLoads;
  __shared__ __attribute__((aligned(1024))) char s_k[2][ST::kBytes];
  __shared__ __attribute__((aligned(1024))) char s_v[2][ST::kBytes];
  __shared__ int s_odd, s_last;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n32 = lane & 31, half = lane >> 5;
  const int D = a.dim, H = a.heads, G = a.group;
  const int rowb = FMT == 0 ? 2 * D : (FMT == 1 ? D : D / 2), nb = D / 32;
  const int capacity = a.b.max_pages << a.page_shift, pmask = (1 << a.page_shift) - 1;

  // the task: heads vary fastest (a head's workgroups on one XCD, where eight
  // divides their number), then parts, then tasks, a sequence's last first
  const int h = blockIdx.x % H, rest = blockIdx.x / H, part = rest % parts, task = rest / parts;
  int s = -1, base = 0;
  for (int s0 = 0; s0 < a.b.n_seq; s0 += 64) {
    int nq = 0;
    if (s0 + lane < a.b.n_seq) nq = (load_seq(a.b, s0 + lane, capacity).n * G + kTaskRows - 1) / kTaskRows;
    const int sum = wave_scan(nq);
    const int before = __popcll(__ballot(base + sum <= task));
    if (before < 64) {
      s = s0 + before;
      base += before ? __builtin_amdgcn_readlane(sum, before - 1) : 0;
      break;
    }
    base += __builtin_amdgcn_readlane(sum, 63);
  }
  if (s < 0 || s >= a.b.n_seq) return;
  const Seq q = load_seq(a.b, s, capacity);
  const int rows = q.n * G, nqt = (rows + kTaskRows - 1) / kTaskRows;
  const int r0 = (nqt - 1 - (task - base)) * kTaskRows, nrow = min(kTaskRows, rows - r0);
  const int pos0 = q.len - q.n;
  auto sees_to = [&](int r) { return max(0, pos0 + r / G + 1); };
  auto sees_from = [&](int r) { return a.window > 0 ? max(0, pos0 + r / G + 1 - a.window) : 0; };
  const int hi_max = sees_to(r0 + nrow - 1), lo_min = sees_from(r0);
  const int hi_min = sees_to(r0), lo_max = sees_from(r0 + nrow - 1);

  const int t_first = lo_min / KT, n_tiles = max(0, (hi_max + KT - 1) / KT - t_first);
  const int used = max(1, min(parts, n_tiles / kMinPart));  // parts with work
  if (part >= used) return;
  const int per_part = (n_tiles + used - 1) / used;
  const int ta = t_first + part * per_part, tb = min(t_first + n_tiles, ta + per_part);

  // this wave's rows
  const int wr0 = r0 + 32 * wave, wrow = min(32, r0 + nrow - wr0);  // (possibly none)
  const bool ok = n32 < wrow;
  const int my_r = ok ? wr0 + n32 : r0, my_i = my_r / G;
  const uint16_t* qp = a.q + (int64_t(q.first) + my_i) * a.q_stride + int64_t(h * G + (my_r - my_i * G)) * D;
  u32x4 qf[DP / 16];
#pragma unroll
  for (int j = 0; j < DP / 16; ++j) {
    const int c = 16 * j + 8 * half;
    qf[j] = u32x4{0, 0, 0, 0};
    if (ok && c < D) qf[j] = *reinterpret_cast<const u32x4*>(qp + c);
  }
  const int hi = ok ? sees_to(my_r) : 0, lo = ok ? sees_from(my_r) : 0;
  const int w_hi_max = wrow > 0 ? sees_to(wr0 + wrow - 1) : 0, w_lo_min = wrow > 0 ? sees_from(wr0) : 0;
  const int w_hi_min = wrow > 0 ? sees_to(wr0) : 0, w_lo_max = wrow > 0 ? sees_from(wr0 + wrow - 1) : 0;

  f32x16 o[CB];
#pragma unroll
  for (int c = 0; c < CB; ++c)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[c][i] = 0.0f;
  float m = -INFINITY, l = 0.0f;

  // staging: this thread's chunks of a tile
  const int32_t* table = a.b.page_table + int64_t(s) * a.b.max_pages;
  u32x4 rk[NL], rv[NL];
  uint32_t sk[NL], sv[NL];
  int pg[NL];
  auto chunk_of = [&](int p, int& tok, int& cc) {
    const int idx = tid + kThreads * p;
    tok = idx / ST::kPer, cc = idx % ST::kPer;
    return ST::kTotal % kThreads == 0 || idx < ST::kTotal;
  };
  auto pages = [&](int t) {  // the pages of tile t's chunks (past the end: of the last token)
#pragma unroll
    for (int p = 0; p < NL; ++p) {
      int tok, cc;
      chunk_of(p, tok, cc);
      pg[p] = table[min(t * KT + min(tok, KT - 1), max(hi_max - 1, 0)) >> a.page_shift];
    }
  };
  auto load = [&](int t) {
#pragma unroll
    for (int p = 0; p < NL; ++p) {
      int tok, cc;
      const bool in = chunk_of(p, tok, cc);
      const int at = min(t * KT + min(tok, KT - 1), max(hi_max - 1, 0)), c = cc * ST::kChunk < D ? cc * ST::kChunk : 0;
      const int page = pg[p] < 0 || pg[p] >= a.n_pages ? 0 : pg[p];
      const int64_t row = ((int64_t(page) * H + h) << a.page_shift) + (at & pmask);
      const int64_t off = row * rowb + (FMT == 0 ? 2 * c : (FMT == 1 ? c : c / 2));
      if (in) {
        rk[p] = *reinterpret_cast<const u32x4*>(a.k + off);
        rv[p] = *reinterpret_cast<const u32x4*>(a.v + off);
        if constexpr (FMT != 0) sk[p] = a.ks[row * nb + c / 32], sv[p] = a.vs[row * nb + c / 32];
      }
      if (pg[p] != page) sk[p] = 1u << 16;  // no such page: what sees it becomes NaN
      else if constexpr (FMT == 0) sk[p] = 0;
    }
  };
  auto store = [&](int t, int buf) {
    const bool edge = t * KT + KT > hi_min || t * KT < lo_max;
    bool odd = false;
#pragma unroll
    for (int p = 0; p < NL; ++p) {
      int tok, cc;
      if (!chunk_of(p, tok, cc)) continue;
      const int at = t * KT + tok;
      const bool none = cc * ST::kChunk >= D;  // channels that pad the tile
      const bool gone = (sk[p] >> 16) != 0;
#pragma unroll
      for (int i = 0; i < ST::kChunk / 8; ++i) {
        const uint32_t wk[4] = {rk[p][0], rk[p][1], rk[p][2], rk[p][3]}, wv[4] = {rv[p][0], rv[p][1], rv[p][2], rv[p][3]};
        uint32_t k4[4], v4[4];
        decode_words<FMT, T>(wk, i, FMT ? scale_of(sk[p] & 255u) : 1.0f, k4);
        decode_words<FMT, T>(wv, i, FMT ? scale_of(sv[p]) : 1.0f, v4);
        if (none || (edge && at >= hi_max)) {
#pragma unroll
          for (int e = 0; e < 4; ++e) k4[e] = v4[e] = 0;
        } else if (gone) {
#pragma unroll
          for (int e = 0; e < 4; ++e) k4[e] = 0x7fff7fffu, v4[e] = 0;
        }
        if (edge) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t fm = finite_mask<T>(v4[e]);
            odd |= fm != 0xffffffffu;
            v4[e] &= fm;
          }
        }
        const int c8 = cc * (ST::kChunk / 8) + i;
        *reinterpret_cast<u32x4*>(&s_k[buf][k_place<DP>(tok, c8)]) = u32x4{k4[0], k4[1], k4[2], k4[3]};
        *reinterpret_cast<u32x4*>(&s_v[buf][v_place<DP>(tok, c8)]) = u32x4{v4[0], v4[1], v4[2], v4[3]};
      }
    }
    if (odd) s_odd = 1;
  };

  if (tid == 0) s_odd = 0;
  __syncthreads();
  if (ta < tb) {
    pages(ta);
    load(ta);
    if (ta + 1 < tb) pages(ta + 1);
    store(ta, 0);
    if (ta + 1 < tb) load(ta + 1);
    if (ta + 2 < tb) pages(ta + 2);
  }
  __syncthreads();

  const uint32_t k_at = k_place<DP>(n32, half);
  const uint32_t v_at = v_place<DP>(4 * half + ((lane >> 2) & 3), 2 * ((lane >> 4) & 1)) + 8 * (lane & 3);
  for (int t = ta; t < tb; ++t) {
    const int buf = (t - ta) & 1, tok0 = t * KT;
    if (tok0 < w_hi_max && tok0 + KT > w_lo_min) {
      const char* kb = s_k[buf];
      const char* vb = s_v[buf];
      f32x16 sc[NB];
#pragma unroll
      for (int b = 0; b < NB; ++b) {
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[b][i] = 0.0f;
#pragma unroll
        for (int j = 0; j < DP / 16; ++j) {
          const u32x4 kf = *reinterpret_cast<const u32x4*>(kb + ((k_at ^ uint32_t(j << 5)) + b * (32 * 2 * DP)));
          sc[b] = T::mfma32(kf, qf[j], sc[b]);
        }
      }
      const bool edge = tok0 + KT > w_hi_min || tok0 < w_lo_max;
      if (edge) {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int tok = tok0 + 32 * b + 8 * (i >> 2) + 4 * half + (i & 3);
            if (tok >= hi || tok < lo) sc[b][i] = -INFINITY;
          }
      }
      float top = -INFINITY;
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, sc[b][i]);
      if (__ballot(top * a.scale > m + 8.0f)) {
        top = fmaxf(top, __shfl_xor(top, 32));
        const float now = fmaxf(m, top * a.scale);
        const float f = m == now ? 1.0f : exp2f(m - now);
        m = now;
        l *= f;
#pragma unroll
        for (int c = 0; c < CB; ++c)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[c][i] *= f;
      }
      const float off = (m == -INFINITY ? 0.0f : -m) + T::kLift;
      uint32_t pw[NB][8];
#pragma unroll
      for (int b = 0; b < NB; ++b) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          sc[b][i] = __builtin_amdgcn_exp2f(fmaf(sc[b][i], a.scale, off));
          l += sc[b][i];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) pw[b][i] = T::pack(sc[b][2 * i], sc[b][2 * i + 1]);
      }
      auto column = [&](int c, int st) {
        const char* p = vb + ((v_at ^ uint32_t(c << 6)) + st * (16 * 2 * DP));
        const u32x2 x = lds_read_transposed(p), y = lds_read_transposed(p + 8 * 2 * DP);
        return u32x4{x[0], x[1], y[0], y[1]};
      };
#pragma unroll
      for (int st = 0; st < 2 * NB; ++st) {
        const uint32_t* w = &pw[st >> 1][4 * (st & 1)];
#pragma unroll
        for (int c = 0; c < CB; ++c) o[c] = T::mfma32(column(c, st), u32x4{w[0], w[1], w[2], w[3]}, o[c]);
      }
    }
    if (t + 1 < tb) {
      store(t + 1, buf ^ 1);
      if (t + 2 < tb) load(t + 2);
      if (t + 3 < tb) pages(t + 3);
    }
    __syncthreads();
  }

  if (__builtin_expect(s_odd, 0)) {  // (as in attn_rows_kernel)
    for (int t = ta; t < tb; ++t) {
      const int tok0 = t * KT;
      if (!(tok0 + KT > hi_min || tok0 < lo_max)) continue;
      for (int tok = max(tok0, lo_min); tok < min(tok0 + KT, hi_max); ++tok) {
        const int64_t row = cached_row(a, table, h, tok);
        if (row < 0) continue;
        const bool sees = tok < hi && tok >= lo;
        const int c0 = fresh(4 * half);
#pragma unroll
        for (int c = 0; c < CB; ++c)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[c][i] += not_finite_value<FMT, T>(a, row, c0 + 32 * c + 8 * (i >> 2) + (i & 3), sees);
      }
    }
  }
  l += __shfl_xor(l, 32);
  if (q.bad) l = __builtin_nanf("");
  uint16_t* dst = a.out + (int64_t(q.first) + my_i) * a.out_stride + int64_t(h * G + (my_r - my_i * G)) * D;
  if (used == 1) {
    const float inv = pos0 + my_i < 0 && l == 0.0f ? 0.0f : 1.0f / l;
    if (ok) {
#pragma unroll
      for (int c = 0; c < CB; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int ch = 32 * c + 8 * i + 4 * half;
          if (ch < D)
            *reinterpret_cast<u32x2*>(dst + ch) = u32x2{T::pack(o[c][4 * i] * inv, o[c][4 * i + 1] * inv), T::pack(o[c][4 * i + 2] * inv, o[c][4 * i + 3] * inv)};
        }
    }
    return;
  }
  // The task's parts: the last workgroup to arrive sums them, in part order.
  const int id = task * H + h;
  const int64_t slot0 = int64_t(id) * parts;
  float* mine = a.part + (slot0 + part) * (kTaskRows * DP) + (32 * wave + n32) * DP;
  float* ml = a.part_ml + (slot0 + part) * (2 * kTaskRows) + 32 * wave + n32;
  if (ok) {
#pragma unroll
    for (int c = 0; c < CB; ++c)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int ch = 32 * c + 8 * (i >> 2) + 4 * half + (i & 3);
        if (ch < D) qtea_detail::store_coherent(mine + ch, o[c][i]);
      }
    if (half == 0) {
      qtea_detail::store_coherent(ml, m);
      qtea_detail::store_coherent(ml + kTaskRows, l);
    }
  }
  __builtin_amdgcn_s_waitcnt(0);  // the part is complete before its arrival is counted
  __syncthreads();
  if (tid == 0) {
    const uint32_t before = __hip_atomic_fetch_add(a.counters + id, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    const bool last = before == uint32_t(used - 1);
    if (last) __hip_atomic_store(a.counters + id, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    s_last = last;
  }
  __syncthreads();
  if (!s_last) return;
  for (int e = tid; e < nrow * (DP / 4); e += kThreads) {
    const int row = e / (DP / 4), ch = (e % (DP / 4)) * 4;
    if (ch >= D) continue;
    float M = -INFINITY, L = 0.0f;
    f32x4 acc = {0, 0, 0, 0};
    for (int w = 0; w < used; ++w) {
      const float* pm = a.part_ml + (slot0 + w) * (2 * kTaskRows) + row;
      const float* po = a.part + (slot0 + w) * (kTaskRows * DP) + row * DP + ch;
      const float mw = qtea_detail::load_coherent(pm), lw = qtea_detail::load_coherent(pm + kTaskRows);
      f32x4 ow;
#pragma unroll
      for (int i = 0; i < 4; ++i) ow[i] = qtea_detail::load_coherent(po + i);
      const float now = fmaxf(M, mw);
      const float fa = M == now ? 1.0f : exp2f(M - now), fb = mw == now ? 1.0f : exp2f(mw - now);
      M = now;
      L = L * fa + lw * fb;
      acc = acc * fa + ow * fb;
    }
    const int r = r0 + row, i = r / G;
    const float inv = pos0 + i < 0 && L == 0.0f ? 0.0f : 1.0f / L;
    uint16_t* to = a.out + (int64_t(q.first) + i) * a.out_stride + int64_t(h * G + (r - i * G)) * D + ch;
    *reinterpret_cast<u32x2*>(to) = u32x2{T::pack(acc[0] * inv, acc[1] * inv), T::pack(acc[2] * inv, acc[3] * inv)};
  }
}

int device_cus() {
  static std::atomic<int> known[qtea_detail::kMaxDevices];
  return qtea_detail::per_current_device(known, [](int dev) {
    int n = 0;
    return hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) == hipSuccess ? n : 0;
  });
}

// The workspace: counters, the parts' maxima and sums, the parts; for the
// grid of the one kernel with two parts a workgroup, and for as many
// workgroups of the other, one part each.
constexpr int kRowsMax = 32;
struct WsLayout {
  int64_t ml, part, bytes;
};
int padded_dim(int dim) { return dim <= 64 ? 64 : (dim <= 128 ? 128 : 256); }
WsLayout ws_layout(int dim, int cus) {
  const int64_t grid = int64_t(cus) * kWgPerCu;
  static_assert(kTaskRows >= 2 * kRowsMax, "the workspace holds either kernel's parts");
  WsLayout w;
  w.ml = (4 * grid + 255) / 256 * 256;
  w.part = w.ml + grid * 2 * kTaskRows * 4;
  w.bytes = w.part + grid * kTaskRows * padded_dim(dim) * 4;
  return w;
}

}  // namespace
}  // namespace qtea_serve

using namespace qtea_serve;

extern "C" {

int qtea_attention_workspace_bytes(int n_q_heads, int head_dim, int64_t* out_bytes) {
  if (!out_bytes || n_q_heads < 1 || head_dim < 32 || head_dim > QTEA_KV_MAX_DIM || head_dim % 32 != 0) return QTEA_ERR_INVALID_ARG;
  const int cus = device_cus();
  if (!cus) return QTEA_ERR_HIP;
  *out_bytes = ws_layout(head_dim, cus).bytes;
  return QTEA_OK;
}

int qtea_paged_attention(const qtea_kv_cache* cache, const qtea_kv_batch* batch, const void* q, void* out, int type,
                         int n_q_heads, int64_t q_stride, int64_t out_stride, float scale, int window, void* workspace,
                         int64_t workspace_bytes, void* stream) {
  if (!cache_ok(cache) || !batch_ok(batch, cache->page_size) || !q || !out || !workspace) return QTEA_ERR_INVALID_ARG;
  if (type != QTEA_F16 && type != QTEA_BF16) return QTEA_ERR_INVALID_ARG;
  if ((cache->format == QTEA_KV_F16 && type != QTEA_F16) || (cache->format == QTEA_KV_BF16 && type != QTEA_BF16)) return QTEA_ERR_INVALID_ARG;
  const int D = cache->head_dim, H = cache->n_heads;
  if (n_q_heads < H || n_q_heads % H != 0 || n_q_heads > 65535) return QTEA_ERR_INVALID_ARG;
  const int64_t width = int64_t(n_q_heads) * D;
  if (q_stride < width || out_stride < width || q_stride % 8 != 0 || out_stride % 8 != 0) return QTEA_ERR_INVALID_ARG;
  if (q_stride > (INT64_MAX >> 34) || out_stride > (INT64_MAX >> 34)) return QTEA_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(out) || !aligned16(workspace)) return QTEA_ERR_INVALID_ARG;
  if (!(scale > 0.0f) || !(scale <= 3.0e38f) || window < 0) return QTEA_ERR_INVALID_ARG;
  const int G = n_q_heads / H;
  const int64_t rows = batch->n_tokens * G;
  const int64_t most_units = (int64_t(batch->max_pages) * cache->page_size + kUnit - 1) / kUnit;
  if (rows > INT32_MAX || (rows / 16 + batch->n_seq) > INT32_MAX / most_units / H) return QTEA_ERR_INVALID_ARG;
  const int cus = device_cus();
  if (!cus) return QTEA_ERR_HIP;
  const WsLayout wl = ws_layout(D, cus);
  if (workspace_bytes < wl.bytes) return QTEA_ERR_WORKSPACE;
  if (batch->n_tokens == 0) return QTEA_OK;
  AttnArgs a;
  a.k = static_cast<const uint8_t*>(cache->k), a.v = static_cast<const uint8_t*>(cache->v);
  a.ks = cache->k_scale, a.vs = cache->v_scale;
  a.q = static_cast<const uint16_t*>(q), a.out = static_cast<uint16_t*>(out);
  a.q_stride = q_stride, a.out_stride = out_stride;
  a.b = kernel_batch(batch);
  a.heads = H, a.group = G, a.dim = D, a.page_shift = log2_of(cache->page_size), a.n_pages = int32_t(cache->n_pages), a.window = window;
  a.scale = scale * 1.44269504088896341f;
  char* ws = static_cast<char*>(workspace);
  a.counters = reinterpret_cast<uint32_t*>(ws);
  a.part_ml = reinterpret_cast<float*>(ws + wl.ml);
  a.part = reinterpret_cast<float*>(ws + wl.part);
  const dim3 block(kThreads);
  const hipStream_t st = static_cast<hipStream_t>(stream);
  // The kernel by a sequence's rows on average (a call's lengths are only known on the device).
  const bool many = rows > int64_t(kRowsMax) * batch->n_seq, two = D <= 128 && rows > int64_t(16) * batch->n_seq;
  const int64_t tasks = rows / kTaskRows + batch->n_seq, grid = int64_t(cus) * kWgPerCu;  // (tasks per head, at most)
  const int parts = int(std::max<int64_t>(1, std::min<int64_t>(grid / (tasks * H), kMaxParts)));
  if (many && tasks * H * parts > INT32_MAX) return QTEA_ERR_INVALID_ARG;
  auto launch = [&](auto dp, auto fmt, auto ty) {
    constexpr int DP = decltype(dp)::value, FMT = decltype(fmt)::value;
    using T = decltype(ty);
    if (many) {
      hipLaunchKernelGGL((attn_tile_kernel<DP, FMT, T>), dim3(uint32_t(tasks * H * parts)), block, 0, st, a, parts);
      return;
    }
    if constexpr (DP <= 128) {
      if (two) {
        hipLaunchKernelGGL((attn_rows_kernel<DP, FMT, T, 2>), dim3(uint32_t(grid)), block, 0, st, a);
        return;
      }
    }
    hipLaunchKernelGGL((attn_rows_kernel<DP, FMT, T, 1>), dim3(uint32_t(grid)), block, 0, st, a);
  };
  auto with_type = [&](auto dp, auto fmt) {
    if (type == QTEA_F16) launch(dp, fmt, F16());
    else launch(dp, fmt, BF16());
  };
  auto with_format = [&](auto dp) {
    if (cache->format == QTEA_KV_E4M3) with_type(dp, std::integral_constant<int, 1>());
    else if (cache->format == QTEA_KV_E2M1) with_type(dp, std::integral_constant<int, 2>());
    else with_type(dp, std::integral_constant<int, 0>());
  };
  const int dp = padded_dim(D);
  if (dp == 64) with_format(std::integral_constant<int, 64>());
  else if (dp == 128) with_format(std::integral_constant<int, 128>());
  else with_format(std::integral_constant<int, 256>());
  return hipGetLastError() == hipSuccess ? QTEA_OK : QTEA_ERR_HIP;
}

}  // extern "C"
