// Causal attention of a batch's newest tokens over the paged cache.
//
// One pass over the cached tokens with a running maximum m and sum l per row
// (a row is a new token and a query head): a tile of tokens gives scores
// s = q . k and weights w = 2^(s c - m), c = scale log2(e), and adds w v to the
// row's sums; m moves only when a score passes it by 8 (the sums are then
// scaled), and the sums are divided by l at the end.  Both products run on the
// matrix cores with the tokens (K, V^T) as the left operand and the rows as
// the right one, so that a score, its weight and the operand of the second
// product are the same register of the same lane: nothing is exchanged
// between lanes on the way.  Quantized values are decoded to `type` by the
// hardware's scaled conversions, which is exact.  Sums, maxima and scores are
// fp32; the weights are rounded to `type` for the second product, as every
// factor of a 16-bit matrix product is (their sum l is not: the result is off
// by one more rounding to `type` at most).
//
// Two kernels, by the rows that a sequence has on average.  Up to 64 (32 past
// 128 channels) the cached bytes bound the call and attn_rows_kernel keeps
// them in registers from the load to the product; beyond, the products do,
// and attn_tile_kernel shares tiles in LDS among 128 rows.  On both sides of the
// line (16 sequences, nine tokens of five query heads a group on average, up
// to 9000 bf16 positions): 89 us against 195.  The choice is the call's: single
// tokens beside a long chunk go to the second kernel with it, whose workgroups
// are few for them.
#include <math.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "serve_common.h"

namespace qtea_serve {
namespace {

constexpr int kTile = 32;      // tokens of one step of a wave (few rows)
constexpr int kWaves = 4, kRowThreads = 64 * kWaves;  // of a workgroup (few rows)
constexpr int kUnit = kTile * kWaves;
constexpr int kThreads = 256;  // of a workgroup of the kernel for many rows
constexpr int kWgPerCu = 2;    // of those

struct AttnArgs {
  const uint8_t* k;
  const uint8_t* v;
  const uint8_t* ks;
  const uint8_t* vs;
  const uint16_t* q;
  uint16_t* out;
  int64_t q_stride, out_stride;  // elements
  Batch b;
  int32_t heads, group, dim, page_shift, n_pages, window, max_slots;
  float scale;       // times log2(e)
  uint32_t* counters;
  float* part;       // partial rows
  float* part_ml;    // their maxima and sums
};

// The first position that a row with `n` positions up to its own sees (n can be
// negative, and the window as large as the type allows).
__device__ __forceinline__ int seen_from(const AttnArgs& a, int n) { return a.window > 0 ? max(0, max(0, n) - a.window) : 0; }

// ---------------------------------------------------------------------------
// Few rows: a task is one sequence, one key/value head and up to 16 R rows
// (new tokens x the query heads that share the head).  A task's tokens are
// split into chunks, one to a workgroup, so that every CU has its workgroups
// busy for about as long; a chunk's tokens are dealt to the waves, 32 at a
// time, and each wave keeps its own sums until the end.  (Equal runs of units
// whatever task they are of balance better but have workgroups change tasks:
// 76 us against 73 for 16 ragged sequences, 49 against 34 for four with drafts.)
//
// A lane's loads: of K, channels of one token, 64 contiguous bytes of it per
// four lanes (the order of the channels is free, as the queries have it too);
// of V, DP / 16 neighbouring channels of 8 tokens, a token's row being the 16
// lanes of a group.  V's pairs of channels per token become pairs of tokens
// per channel by one byte permutation a word.
//
// Bound by HBM for long histories (one token over 260001 positions in E2M1,
// 283 MB: 61 us; 16 tokens over up to 16000 in E4M3, 360 MB: 73 us; each
// further byte at 5.7 to 6.6 TB/s, of 7.1 that a plain read reaches, beside 15
// to 18 us for the start and the join), below that by the chain of dependent
// reads: lengths, pages, values, parts (one token over 700: 10.5 us, of which
// 1.1 are the launch, 1.5 the chunk search, 1.1 the pages, 2 the one tile, 0.9
// the waves' join, 3 the arrival and the parts).  A wave of 32 rows reads
// each value once, which is faster than two waves of 16 that read it from the
// L1 and L2 (34 us against 53 for four sequences' drafts).
// ---------------------------------------------------------------------------

// The work of sequence s: `nqt` row tasks per head, each of `cnt` units of
// tokens from unit t0 on (the same for all: what its first row sees starts
// there, what the last one sees ends there).
struct SeqWork {
  Seq q;
  int t0, cnt, nqt, tasks;
};

template <int MT>
__device__ __forceinline__ SeqWork seq_work(const AttnArgs& a, int s) {
  SeqWork w;
  w.q = load_seq(a.b, s, a.b.max_pages << a.page_shift);
  const int first = w.q.len - w.q.n + 1;  // positions the first row's prefix holds
  const int lo = seen_from(a, first);
  w.t0 = lo / kUnit;
  w.cnt = max(1, (w.q.len + kUnit - 1) / kUnit - w.t0);
  w.nqt = (w.q.n * a.group + MT - 1) / MT;
  w.tasks = w.nqt * a.heads;
  return w;
}

// Chunks of a task of cnt units, for chunks of about 1 / rate units.
__device__ __forceinline__ int chunks_of(int cnt, float rate) { return max(1, int(__builtin_ceilf(float(cnt) * rate))); }

// Inclusive sum over the wave's lanes.
__device__ __forceinline__ int wave_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);  // from 1, 2, 4, 8 lanes below in the row of 16
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // a row's last lane to the next row
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // lane 31 to the upper half
  return x;
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
  static constexpr int kScaleWords = DP <= 128 ? 1 : 2;                     // words of a token's K scales
  uint32_t k[2][kKWords];
  uint32_t v[8][kVWords];
  uint32_t ks[2][kScaleWords];  // scale bytes of the token, block b in byte b
  uint32_t vs[8];               // the word of the token's scale bytes that holds this lane's
};

template <int N>
__device__ __forceinline__ void load_words(const uint8_t* p, uint32_t* w) {
  if constexpr (N % 4 == 0) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const u32x4 x = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p + 4 * i));
#pragma unroll
      for (int j = 0; j < 4; ++j) w[i + j] = x[j];
    }
  } else if constexpr (N == 2) {
    const u32x2 x = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(p));
    w[0] = x[0], w[1] = x[1];
  } else {
    w[0] = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(p));
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

// Channels 2 i, 2 i + 1 of the codes in w.
template <int FMT, class T>
__device__ __forceinline__ uint32_t decode_pair(const uint32_t* w, int i, float s) {
  if constexpr (FMT == 0) return w[i];
  else if constexpr (FMT == 1) return i % 2 ? T::template e4m3<true>(w[i / 2], s) : T::template e4m3<false>(w[i / 2], s);
  else {
    switch (i % 4) {
      case 0: return T::template e2m1<0>(w[i / 4], s);
      case 1: return T::template e2m1<1>(w[i / 4], s);
      case 2: return T::template e2m1<2>(w[i / 4], s);
      default: return T::template e2m1<3>(w[i / 4], s);
    }
  }
}

// The factor of the scale byte at bit `shift` of a word.
__device__ __forceinline__ float scale_at(uint32_t word, int shift) { return scale_of(__builtin_amdgcn_ubfe(word, shift, 8)); }

// A 16-bit channel pair is not finite in either half.
template <class T>
__device__ __forceinline__ uint32_t finite_mask(uint32_t x) {
  const uint32_t lo = (x & T::kExp) == T::kExp ? 0u : 0xffffu;
  const uint32_t hi = ((x >> 16) & T::kExp) == T::kExp ? 0u : 0xffff0000u;
  return lo | hi;
}

// The largest scale byte under which no code passes the type's range.
template <int FMT, class T>
constexpr uint32_t kFiniteScale = (T::kExp == 0x7c00u ? 15 : 127) - (FMT == 1 ? 8 : 2) + 127;

// Zeroes the values of N words of V codes that are not finite; whether there
// were any.  (E4M3: NaN codes; blocks of a NaN scale; codes that a large scale
// takes past the type's range, which are looked for where there is such a scale.)
template <int FMT, class T, int N>
__device__ __forceinline__ bool drop_not_finite(uint32_t* w, uint32_t& scales, int shift) {
  uint32_t keep_all = 0xffffffffu, lost = 0;
  bool large = false;
  if constexpr (FMT != 0) {
    const uint32_t scale = __builtin_amdgcn_ubfe(scales, shift, 8);
    keep_all = scale == 255u ? 0u : 0xffffffffu;
    large = scale > kFiniteScale<FMT, T> && scale != 255u;
    scales &= keep_all;
    lost = ~keep_all;
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    uint32_t keep = keep_all;
    if constexpr (FMT == 0) keep = finite_mask<T>(w[i]);
    if constexpr (FMT == 1) {
      const uint32_t nan = (((w[i] & 0x7f7f7f7fu) + 0x01010101u) >> 7) & 0x01010101u;  // per byte: all ones below the sign
      keep &= ~(nan * 255u);
    }
    lost |= ~keep;
    w[i] &= keep;
  }
  if constexpr (FMT != 0) {
    if (__builtin_expect(__ballot(large) != 0, 0)) {
      constexpr int kPairs = FMT == 1 ? 2 : 4, kBits = FMT == 1 ? 8 : 4;  // of a word's codes
#pragma unroll
      for (int i = 0; i < kPairs * N; ++i) {
        const uint32_t fm = finite_mask<T>(decode_pair<FMT, T>(w, i, scale_at(scales, shift)));
        const uint32_t codes = ((fm & 0xffffu ? 0u : 1u) | (fm >> 16 ? 0u : 1u << kBits)) * ((1u << kBits) - 1);  // those to drop
        lost |= codes;
        w[i / kPairs] &= ~(codes << (2 * kBits * (i % kPairs)));
      }
    }
  }
  return lost != 0;
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

// Channel c of a cached V row if it is not finite, else 0 (for the sum of a row
// that sees it: a positive weight does not change it).
template <int FMT, class T>
__device__ __forceinline__ float not_finite_value(const AttnArgs& a, int64_t row, int c) {
  c = min(c, a.dim - 1);  // (sums of channels past the last are not used)
  uint32_t w;
  if constexpr (FMT == 0) w = reinterpret_cast<const uint16_t*>(a.v)[row * a.dim + c];
  else if constexpr (FMT == 1) w = T::template e4m3<false>(a.v[row * a.dim + c], scale_of(a.vs[row * (a.dim / 32) + c / 32]));
  else w = T::template e2m1<0>(uint32_t(a.v[row * (a.dim / 2) + c / 2]) >> (4 * (c & 1)), scale_of(a.vs[row * (a.dim / 32) + c / 32]));
  const float v = float(__builtin_bit_cast(typename T::pair, w)[0]);
  return fabsf(v) < INFINITY ? 0.0f : v;
}

__device__ __forceinline__ void store_coherent2(float* p, float x, float y) {
  const f32x2 v = {x, y};
  __hip_atomic_store(reinterpret_cast<uint64_t*>(p), __builtin_bit_cast(uint64_t, v), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ f32x2 load_coherent2(const float* p) {
  return __builtin_bit_cast(f32x2, __hip_atomic_load(reinterpret_cast<uint64_t*>(const_cast<float*>(p)), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}

// A row's running maximum, sum and four channels, and those of other tokens.
struct Joined {
  float M = -INFINITY, L = 0.0f;
  f32x4 acc = {0, 0, 0, 0};
  __device__ __forceinline__ void add(float m, float l, f32x4 o) {
    const float now = fmaxf(M, m);
    const float fa = M == now ? 1.0f : __builtin_amdgcn_exp2f(M - now), fb = m == now ? 1.0f : __builtin_amdgcn_exp2f(m - now);
    M = now;
    L = L * fa + l * fb;
    acc = acc * fa + o * fb;
  }
};

// Counts this workgroup's arrival; whether it is the last of n.
__device__ __forceinline__ bool last_to_arrive(uint32_t* counter, int n, int* s_last) {
  asm volatile("" ::: "memory");  // (no store moves past the wait)
  __builtin_amdgcn_s_waitcnt(0);  // what it stored is complete before its arrival is counted
  asm volatile("" ::: "memory");
  __syncthreads();
  if (threadIdx.x == 0) {
    const uint32_t before = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    const bool last = before == uint32_t(n - 1);
    if (last) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    *s_last = last;
  }
  __syncthreads();
  return *s_last;
}

constexpr int kJoin = 12;  // parts joined at once
constexpr int kCounterWords = 32;  // a line a counter: arrivals at one line are served one after another

// Joins the parts of a task's rows in part order, by the whole workgroup: four
// channels a thread, and with few rows the parts dealt to groups of threads,
// whose results are joined in group order.  The parts are `step` slots apart.
// `give(row, channel, result)` takes the results.  `lds`: 6 floats a thread.  Every load of a
// batch is on its way before the first is used: they come from the other
// XCDs' stores, past this one's L2.
template <int DP, int MT, int THREADS, class Give>
__device__ __forceinline__ void join_parts(const AttnArgs& a, const float* part_ml, int64_t slot0, int step, int n_parts, int nrow, float* lds, Give give) {
  constexpr int kBatch = 8;
  const int tid = threadIdx.x;
  const int quads = a.dim / 4, items = nrow * quads;
  const int groups = max(1, min(THREADS / items, n_parts)), grp = groups > 1 ? tid / items : 0;
  for (int e = tid - grp * items; e < items && grp < groups; e += groups > 1 ? items : THREADS) {
    const int row = e / quads, ch = (e - row * quads) * 4;
    Joined j;
    for (int w0 = grp; w0 < n_parts; w0 += groups * kBatch) {
      float mw[kBatch], lw[kBatch];
      f32x2 x[kBatch], y[kBatch];
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        const int64_t sl = slot0 + step * min(w0 + groups * i, n_parts - 1);
        const float* pm = part_ml + sl * (2 * MT) + row;
        const float* po = a.part + sl * (MT * DP) + row * DP + ch;
        mw[i] = qtea_detail::load_coherent(pm), lw[i] = qtea_detail::load_coherent(pm + MT);
        x[i] = load_coherent2(po), y[i] = load_coherent2(po + 2);
      }
#pragma unroll
      for (int i = 0; i < kBatch; ++i)
        if (w0 + groups * i < n_parts) j.add(mw[i], lw[i], f32x4{x[i][0], x[i][1], y[i][0], y[i][1]});
    }
    if (groups > 1) {
      *reinterpret_cast<f32x4*>(lds + 4 * tid) = j.acc;
      lds[4 * THREADS + 2 * tid] = j.M, lds[4 * THREADS + 2 * tid + 1] = j.L;
    } else {
      give(row, ch, j);
    }
  }
  if (groups > 1) {
    __syncthreads();
    if (tid < items) {
      Joined j;
      for (int k = 0; k < groups; ++k) {
        const int t = tid + k * items;
        j.add(lds[4 * THREADS + 2 * t], lds[4 * THREADS + 2 * t + 1], *reinterpret_cast<const f32x4*>(lds + 4 * t));
      }
      const int row = tid / quads;
      give(row, (tid - row * quads) * 4, j);
    }
  }
}

constexpr int lds_width(int DP) { return DP < 128 ? DP : 128; }  // channels joined at a time

constexpr float kMinUnits = 2.0f;  // of a chunk: what joining two costs
// Workgroups per CU, each of one wave per SIMD: as many as have the registers
// for a tile on the way beside their sums.
constexpr int rows_per_cu(int DP, int FMT, int R) { return R * DP >= 256 ? 1 : ((FMT == 0 && R * DP == 128) || R == 2 ? 2 : 3); }

// EX: the heads have DP channels; else they have fewer, and what lies past
// them is read from the first channels instead (queries are 0 there, and sums
// not used).
template <int DP, int FMT, class T, int R, bool EX>
__global__ __launch_bounds__(kRowThreads, rows_per_cu(DP, FMT, R)) void attn_rows_kernel(const AttnArgs a) {
  using TL = Tile<DP, FMT>;
  constexpr int MT = 16 * R;
  constexpr int CH = TL::kCH, CW = lds_width(DP), CS = CW + 4;  // (+ 4: rows on other banks)
  __shared__ float s_o[kWaves][16][CS];
  __shared__ float s_m[kWaves][MT], s_l[kWaves][MT], s_sum[MT];
  __shared__ int s_last, s_odd;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n16 = lane & 15, g = lane >> 4;
  const int D = EX ? DP : a.dim, H = a.heads, G = a.group;
  const uint32_t rowb = FMT == 0 ? 2 * D : (FMT == 1 ? D : D / 2), nb = D / 32;
  const int pmask = (1 << a.page_shift) - 1;
  // where this lane's codes and scales are in a half's rows
  auto code_bytes = [](uint32_t channels) { return FMT == 0 ? 2 * channels : (FMT == 1 ? channels : channels / 2); };
  const uint32_t k_lane = n16 * rowb, k_at = k_lane + code_bytes(!EX && g * TL::kChunk >= D ? 0 : g * TL::kChunk);
  const uint32_t v_at = 4 * g * rowb + code_bytes(!EX && n16 * CH >= D ? 0 : n16 * CH);
  // where this lane's scale bytes are in their words
  const int k_shift = 8 * (g * TL::kChunk / 32), v_shift = 8 * (n16 * CH / 32 % 4);

  __builtin_amdgcn_s_setprio(3);
  // The call's chunks (each wave for itself: no barrier).  Their size: the
  // smallest of 64 candidates, from an equal share of all units for every
  // workgroup to three times that, whose chunks are no more than the
  // workgroups; for more sequences than a wave has lanes, half as much again
  // as the share (what is over waits for a workgroup to be free).
  const bool one_wave = a.b.n_seq <= 64;  // of sequences, a lane each
  SeqWork mine = {};
  int W = 0;  // units of all tasks
  for (int s0 = 0; s0 < a.b.n_seq; s0 += 64) {
    mine = SeqWork{};
    if (s0 + lane < a.b.n_seq) mine = seq_work<MT>(a, s0 + lane);
    W += __builtin_amdgcn_readlane(wave_scan(mine.cnt * mine.tasks), 63);
  }
  const float share = fmaxf(float(W) / float(gridDim.x), kMinUnits);
  float rate = 1.0f / (share * 1.5f);
  if (one_wave) {
    const float r = 1.0f / (share * (1.0f + float(lane) * (2.0f / 63.0f)));
    int chunks = 0;
    for (int j = 0; j < a.b.n_seq; ++j) chunks += __builtin_amdgcn_readlane(mine.tasks, j) * chunks_of(__builtin_amdgcn_readlane(mine.cnt, j), r);
    const uint64_t fit = __ballot(chunks <= int(gridDim.x));
    rate = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(r), fit ? __builtin_ctzll(fit) : 63));
  }

  for (int id = blockIdx.x;; id += gridDim.x) {
    // this chunk's sequence; chunks of split tasks before it have the first slots
    int s = -1, base = 0, slot0 = 0;
    SeqWork sw;
    for (int s0 = 0; s0 < a.b.n_seq; s0 += 64) {
      if (!one_wave) {
        mine = SeqWork{};
        if (s0 + lane < a.b.n_seq) mine = seq_work<MT>(a, s0 + lane);
      }
      const int k = chunks_of(mine.cnt, rate), sum = wave_scan(k * mine.tasks), split = wave_scan(k > 1 ? k * mine.tasks : 0);
      const int before = __popcll(__ballot(base + sum <= id));
      if (before < 64) {
        s = s0 + before;
        base += before ? __builtin_amdgcn_readlane(sum, before - 1) : 0;
        slot0 += before ? __builtin_amdgcn_readlane(split, before - 1) : 0;
        auto of = [&](int x) { return __builtin_amdgcn_readlane(x, before); };
        sw = SeqWork{{of(mine.q.first), of(mine.q.n), of(mine.q.len), of(mine.q.bad) != 0}, of(mine.t0), of(mine.cnt), of(mine.nqt), of(mine.tasks)};
        break;
      }
      base += __builtin_amdgcn_readlane(sum, 63);
      slot0 += __builtin_amdgcn_readlane(split, 63);
    }
    if (s < 0 || s >= a.b.n_seq) return;
    const int parts = __builtin_amdgcn_readfirstlane(chunks_of(sw.cnt, rate)), task = (id - base) / parts, part = (id - base) - task * parts;
    const int per = sw.cnt / parts, more = sw.cnt - per * parts;
    const int ua = part * per + min(part, more), ub = ua + per + (part < more ? 1 : 0);  // units [ua, ub) of the task
    // (starts that decrease can make the counts above overflow: not past the operands or the workspace)
    if (task < 0 || task >= sw.tasks || slot0 < 0 || (parts > 1 && slot0 + (task + 1) * parts > a.max_slots)) return;
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
      lo[r] = seen_from(a, pos0 + i + 1);
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
    const int lo_min = seen_from(a, pos0 + i_first + 1), lo_max = seen_from(a, pos0 + i_last + 1);

    f32x4 o[R][CH];
    float m[R], l[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      m[r] = -INFINITY, l[r] = 0.0f;
#pragma unroll
      for (int c = 0; c < CH; ++c) o[r][c] = f32x4{0, 0, 0, 0};
    }
    bool bad = sw.q.bad, odd = false;
    if (tid == 0) s_odd = 0;  // (read after the barriers below)

    const int tile_a = (sw.t0 + ua) * kWaves, tile_b = min((sw.t0 + ub) * kWaves, (hi_max + kTile - 1) / kTile);
    const int32_t* table = a.b.page_table + int64_t(s) * a.b.max_pages;
    // The pages of this wave's next 32 tiles' halves, a lane each (a half past
    // the end repeats the last one).
    int t = tile_a + wave;
    if (t < lo_min / kTile) t += (lo_min / kTile - t + kWaves - 1) / kWaves * kWaves;
    int page = 0, page_at = 0;  // (page_at: the tile of the first lane)
    auto half_first = [&](int t, int sub) { return min(t * kTile + 16 * sub, (hi_max - 1) & ~15); };
    auto load_pages = [&](int from) {
      const int tok = half_first(from + (lane >> 1) * kWaves, lane & 1);
      page = table[tok >> a.page_shift], page_at = from;
      const bool none = page < 0 || page >= a.n_pages;
      // (a half below the window holds no visible token: its page may be gone)
      bad = bad || __ballot(none && tok + 16 > lo_min) != 0;
      if (none) page = 0;
    };
    // Cached rows of the halves' first tokens.
    auto places = [&](int t, int64_t (&prow)[2]) {
      const int k = (t - page_at) / kWaves;
#pragma unroll
      for (int sub = 0; sub < 2; ++sub)
        prow[sub] = ((int64_t(__builtin_amdgcn_readlane(page, 2 * k + sub)) * H + h) << a.page_shift) + (half_first(t, sub) & pmask);
    };
    TL x;
    auto load_k = [&](const int64_t (&prow)[2]) {
#pragma unroll
      for (int sub = 0; sub < 2; ++sub) {
        const uint8_t* kp = a.k + prow[sub] * rowb;
        const uint32_t at = fresh(k_at);
#pragma unroll
        for (int i = 0; i < TL::kChunks; ++i) {
          constexpr int kLoad = TL::kKWords / TL::kChunks;
          const uint8_t* from = kp + at + i * 16 * kLoad;
          if (!EX && i * (4 * TL::kChunk) + g * TL::kChunk >= D) from = kp + k_lane;  // (past the last channel)
          load_words<kLoad>(from, x.k[sub] + i * kLoad);
        }
        if constexpr (FMT != 0) {
          const uint8_t* sp = a.ks + prow[sub] * nb;
          if constexpr (EX) {
            const uint32_t sat = fresh(nb * n16);
            if constexpr (DP == 64) x.ks[sub][0] = *reinterpret_cast<const uint16_t*>(sp + sat);
            else load_words<TL::kScaleWords>(sp + sat, x.ks[sub]);
          } else {
#pragma unroll
            for (int w = 0; w < TL::kScaleWords; ++w) x.ks[sub][w] = 0;
#pragma unroll
            for (int i = 0; i < TL::kChunks; ++i) {
              const int c = i * (4 * TL::kChunk) + g * TL::kChunk;
              x.ks[sub][i * TL::kChunk / 32] |= uint32_t(sp[nb * n16 + uint32_t(c < D ? c : 0) / 32]) << (8 * (i * TL::kChunk / 8 % 4) + k_shift);
            }
          }
        }
      }
    };
    auto load_v = [&](const int64_t (&prow)[2]) {
#pragma unroll
      for (int sub = 0; sub < 2; ++sub) {
        const uint8_t* vp = a.v + prow[sub] * rowb;
        const uint32_t at = fresh(v_at);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if constexpr (FMT == 2 && CH == 4) x.v[4 * sub + j][0] = *reinterpret_cast<const uint16_t*>(vp + at + j * rowb);
          else load_words<TL::kVWords>(vp + at + j * rowb, x.v[4 * sub + j]);
        }
        if constexpr (FMT != 0) {
          const uint8_t* sp = a.vs + prow[sub] * nb;
          if constexpr (EX && DP == 64) {
            uint32_t w[2];
            load_words<2>(sp + uint32_t(fresh(8 * g)), w);
            x.vs[4 * sub] = w[0], x.vs[4 * sub + 1] = w[0] >> 16, x.vs[4 * sub + 2] = w[1], x.vs[4 * sub + 3] = w[1] >> 16;
          } else if constexpr (EX && DP == 128) {
            load_words<4>(sp + uint32_t(fresh(16 * g)), x.vs + 4 * sub);
          } else if constexpr (EX) {
#pragma unroll
            for (int j = 0; j < 4; ++j) load_words<1>(sp + uint32_t(fresh(32 * g + 4 * (n16 >> 3))) + 8 * j, x.vs + 4 * sub + j);
          } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) x.vs[4 * sub + j] = uint32_t(sp[(4 * g + j) * nb + uint32_t(n16 * CH < D ? n16 * CH : 0) / 32]) << v_shift;
          }
        }
      }
    };
    // One tile ahead: the next tile's K is asked for as soon as this one's is
    // used up, its V at this one's end.  (The last tile asks for itself again:
    // a branch here would have the next wait drain every load.)
    int64_t prow[2];
    if (t < tile_b) {
      load_pages(t);
      places(t, prow);
      load_k(prow);
      load_v(prow);
    }
    // (the queries are here before the loop: in it, a wait for them would be one for every load)
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int j = 0; j < TL::kSteps; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) asm volatile("" : "+v"(qf[r][j][e]));
    // A wave gives way as it gets on: of those that wait for memory the oldest
    // would go first, and the youngest start when the others are done.
    const int third = max(1, (tile_b - t + 3 * kWaves - 1) / (3 * kWaves)) * kWaves;  // tiles of its first third
    const int q1 = t + third, q2 = q1 + third;
    __builtin_amdgcn_s_setprio(2);
    for (; t < tile_b; t += kWaves) {
      const int tok0 = t * kTile;
      if (t == q1) __builtin_amdgcn_s_setprio(1);
      if (t == q2) __builtin_amdgcn_s_setprio(0);
      if (t + kWaves < tile_b) {
        if (t + kWaves - page_at >= 32 * kWaves) load_pages(t + kWaves);
        places(t + kWaves, prow);
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
          const int i = j / per;
          decode_words<FMT, T>(x.k[sub], j, FMT ? scale_at(x.ks[sub][i * TL::kChunk / 32], 8 * (i * TL::kChunk / 8 % 4) + k_shift) : 1.0f, kw);
#pragma unroll
          for (int r = 0; r < R; ++r)
            sc[r][sub] = T::mfma16(u32x4{kw[0], kw[1], kw[2], kw[3]}, u32x4{qf[r][j][0], qf[r][j][1], qf[r][j][2], qf[r][j][3]}, sc[r][sub]);
        }
      }
      load_k(prow);
      __builtin_amdgcn_sched_barrier(0);
      const bool edge = tok0 + kTile > hi_min || tok0 < lo_max;
      if (edge) {
        // What a row does not see has no weight; and values that are not
        // finite are left out, since 0 times them is not 0: the rows that see
        // them get them below.
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
        for (int j = 0; j < 8; ++j) {
          const bool found = drop_not_finite<FMT, T, TL::kVWords>(x.v[j], x.vs[j], v_shift);
          odd |= found && tok0 + 16 * (j / 4) + 4 * g + j % 4 < hi_max;
        }
      }
      // softmax: the running maximum moves only when a score passes it by 8 powers of two
      uint32_t pw[R][4];
#pragma unroll
      for (int r = 0; r < R; ++r) {
        if (r > 0 && 16 * r >= nrow) {  // (no such rows)
          pw[r][0] = pw[r][1] = pw[r][2] = pw[r][3] = 0;
          continue;
        }
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
      // V^T (16 of a lane row's channels x 32 tokens) times the weights: pairs
      // of tokens per channel from the tokens' pairs of channels
#pragma unroll
      for (int cp = 0; cp < CH / 2; ++cp) {
        uint32_t vt[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) vt[j] = decode_pair<FMT, T>(x.v[j], cp, FMT ? scale_at(x.vs[j], v_shift) : 1.0f);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          u32x4 w;
#pragma unroll
          for (int jj = 0; jj < 4; ++jj) w[jj] = __builtin_amdgcn_perm(vt[2 * jj + 1], vt[2 * jj], e ? 0x07060302u : 0x05040100u);
#pragma unroll
          for (int r = 0; r < R; ++r) o[r][2 * cp + e] = T::mfma16(w, u32x4{pw[r][0], pw[r][1], pw[r][2], pw[r][3]}, o[r][2 * cp + e]);
        }
      }
      load_v(prow);
      __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_s_setprio(3);
    // this lane's tokens of the sums: over the four lanes of a row
#pragma unroll
    for (int r = 0; r < R; ++r) {
      l[r] += __shfl_xor(l[r], 16);
      l[r] += __shfl_xor(l[r], 32);
      if (bad) l[r] = __builtin_nanf("");
      if (g == 0) s_m[wave][16 * r + n16] = m[r], s_l[wave][16 * r + n16] = l[r];
    }
    __syncthreads();
    if (__builtin_expect(odd, 0)) s_odd = 1;

    // The waves' rows joined: each at the common maximum, summed in wave order.
    const int slot = slot0 + task * parts + part;
    float* to_part = a.part + int64_t(slot) * (MT * DP);
    float* to_ml = a.part_ml + int64_t(slot) * (2 * MT);
    auto give = [&](int row, int ch, f32x4 acc, float L) {
      const int rr = r0 + row, i = rr / G, hh = rr - i * G;
      const float inv = pos0 + i < 0 && L == 0.0f ? 0.0f : 1.0f / L;  // (no position: nothing was summed)
      uint16_t* dst = a.out + (token_row0 + i) * a.out_stride + int64_t(h * G + hh) * D + ch;
      *reinterpret_cast<u32x2*>(dst) = u32x2{T::pack(acc[0] * inv, acc[1] * inv), T::pack(acc[2] * inv, acc[3] * inv)};
    };
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int row = 16 * r + n16;
      float M = s_m[0][row];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) M = fmaxf(M, s_m[w][row]);
      const float f = m[r] == M ? 1.0f : __builtin_amdgcn_exp2f(m[r] - M);
#pragma unroll
      for (int half = 0; half < DP / CW; ++half) {
        if (DP == CW || (4 * g * CH) / CW == half) {
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int c = 0; c < CH; c += 4)
              *reinterpret_cast<f32x4*>(&s_o[wave][n16][(4 * g + i) * CH + c - half * CW]) =
                  f32x4{o[r][c][i] * f, o[r][c + 1][i] * f, o[r][c + 2][i] * f, o[r][c + 3][i] * f};
        }
        if (half == 0 && g == 0 && wave == kWaves - 1) {
          float L = 0.0f;
#pragma unroll
          for (int w = 0; w < kWaves; ++w) L += s_l[w][row] * (s_m[w][row] == M ? 1.0f : __builtin_amdgcn_exp2f(s_m[w][row] - M));
          s_sum[row] = L;
          if (row < nrow && parts > 1) qtea_detail::store_coherent(to_ml + row, M), qtea_detail::store_coherent(to_ml + MT + row, L);
        }
        __syncthreads();
        for (int e = tid; e < min(16, nrow - 16 * r) * (CW / 4); e += kRowThreads) {
          const int rw = e / (CW / 4), c4 = (e % (CW / 4)) * 4, row2 = 16 * r + rw, ch = half * CW + c4;
          if (ch >= D) continue;
          f32x4 acc = *reinterpret_cast<const f32x4*>(&s_o[0][rw][c4]);
#pragma unroll
          for (int w = 1; w < kWaves; ++w) acc += *reinterpret_cast<const f32x4*>(&s_o[w][rw][c4]);
          if (__builtin_expect(s_odd, 0)) {
            // values that are not finite, of the tokens this row sees
            const int i = (r0 + row2) / G;
            const int to = min(tile_b * kTile, max(0, pos0 + i + 1)), from = seen_from(a, pos0 + i + 1);
            for (int tok = max(tile_a * kTile, from); tok < to; ++tok) {
              const int tok0 = tok & ~(kTile - 1);
              const int64_t at = tok0 + kTile > hi_min || tok0 < lo_max ? cached_row(a, table, h, tok) : -1;
              if (at < 0) continue;  // (of another tile: taken with the rest)
#pragma unroll
              for (int e2 = 0; e2 < 4; ++e2) acc[e2] += not_finite_value<FMT, T>(a, at, ch + e2);
            }
          }
          if (parts == 1) {
            give(row2, ch, acc, s_sum[row2]);
          } else {
            store_coherent2(to_part + row2 * DP + ch, acc[0], acc[1]);
            store_coherent2(to_part + row2 * DP + ch + 2, acc[2], acc[3]);
          }
        }
        __syncthreads();
      }
    }
    if (parts > 1) {
      // The last of the task's workgroups to arrive joins their parts, in
      // order; of more than kJoin parts, first the last of every kJoin joins
      // those, into the place of their first (with maxima and sums of their
      // own: other threads may still read the parts').
      float* joined_ml = a.part_ml + int64_t(a.max_slots) * (2 * MT);
      const bool tree = parts > kJoin;
      const int first = slot - part, mine0 = first + (tree ? part / kJoin * kJoin : 0), n_mine = tree ? min(kJoin, first + parts - mine0) : parts;
      if (last_to_arrive(a.counters + mine0 * kCounterWords, n_mine, &s_last)) {
        if (tree) {
          join_parts<DP, MT, kRowThreads>(a, a.part_ml, mine0, 1, n_mine, nrow, &s_o[0][0][0], [&](int row, int ch, const Joined& j) {
            float* at = a.part + int64_t(mine0) * (MT * DP) + row * DP + ch;
            store_coherent2(at, j.acc[0], j.acc[1]);
            store_coherent2(at + 2, j.acc[2], j.acc[3]);
            if (ch == 0) {
              float* ml = joined_ml + int64_t(mine0) * (2 * MT) + row;
              qtea_detail::store_coherent(ml, j.M), qtea_detail::store_coherent(ml + MT, j.L);
            }
          });
          if (last_to_arrive(a.counters + (a.max_slots + first) * kCounterWords, (parts + kJoin - 1) / kJoin, &s_last))
            join_parts<DP, MT, kRowThreads>(a, joined_ml, first, kJoin, (parts + kJoin - 1) / kJoin, nrow, &s_o[0][0][0], [&](int row, int ch, const Joined& j) { give(row, ch, j.acc, j.L); });
        } else {
          join_parts<DP, MT, kRowThreads>(a, a.part_ml, first, 1, parts, nrow, &s_o[0][0][0], [&](int row, int ch, const Joined& j) { give(row, ch, j.acc, j.L); });
        }
      }
      __syncthreads();
    }
  }
}

// ---------------------------------------------------------------------------
// Many rows: a task is one sequence, one key/value head and 128 rows, 32 per
// wave; the workgroup stages tiles of 64 tokens (32 past 128 channels) through
// LDS, decoded, for its four waves: two tiles, one being read while the next
// comes in by way of registers.  Where there are few tasks their tokens are
// split into `parts`.
//
// Bound by instruction issue: for 64 tokens x 32 rows x 128 channels a wave
// issues 32 products (1024 cycles of its SIMD) and about 265 vector
// instructions (1440 cycles, of them 512 for the exponentials), and the two
// waves of a SIMD overlap little of the one with the other: 38 % of the
// cycles have a product in the matrix core, 49 % a vector instruction.  A
// 2048-token chunk over 12345 positions, 32 heads, E4M3: 430 us, 883 TFLOP/s
// (fp16 cache 831, E2M1 917); six prompts of up to 4000 tokens, 64 channels,
// window 1024, bf16: 107 us, 605 TFLOP/s of the pairs in the windows (28 and
// 66 % of the cycles).
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

template <int DP, int FMT, class T, bool EX>  // (EX as above)
__global__ __launch_bounds__(kThreads, DP == 256 ? 1 : 2) void attn_tile_kernel(const AttnArgs a, int parts) {
  using ST = Stage<DP, FMT>;
  constexpr int KT = ST::kTok, NB = ST::kBlocks, CB = DP / 32, NL = ST::kLoads;
  __shared__ __attribute__((aligned(1024))) char s_k[2][ST::kBytes];
  __shared__ __attribute__((aligned(1024))) char s_v[2][ST::kBytes];
  __shared__ int s_odd, s_last;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n32 = lane & 31, half = lane >> 5;
  const int D = EX ? DP : a.dim, H = a.heads, G = a.group;
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
  auto sees_from = [&](int r) { return seen_from(a, pos0 + r / G + 1); };
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
  uint32_t sk[NL] = {}, sv[NL] = {};
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
  // (PLAIN: every token of the tile is one that all rows see, and has a page)
  auto store_as = [&](int t, int buf, auto plain) {
    constexpr bool PLAIN = decltype(plain)::value;
    bool odd = false;
#pragma unroll
    for (int p = 0; p < NL; ++p) {
      int tok, cc;
      if (!chunk_of(p, tok, cc)) continue;
      const bool none = !EX && cc * ST::kChunk >= D;  // channels that pad the tile
      const bool past = !PLAIN && t * KT + tok >= hi_max, gone = !PLAIN && (sk[p] >> 16) != 0;
#pragma unroll
      for (int i = 0; i < ST::kChunk / 8; ++i) {
        const uint32_t wk[4] = {rk[p][0], rk[p][1], rk[p][2], rk[p][3]}, wv[4] = {rv[p][0], rv[p][1], rv[p][2], rv[p][3]};
        uint32_t k4[4], v4[4];
        decode_words<FMT, T>(wk, i, FMT ? scale_of(PLAIN ? sk[p] : sk[p] & 255u) : 1.0f, k4);
        decode_words<FMT, T>(wv, i, FMT ? scale_of(sv[p]) : 1.0f, v4);
        if (none || past) {
#pragma unroll
          for (int e = 0; e < 4; ++e) k4[e] = v4[e] = 0;
        } else if (gone) {
#pragma unroll
          for (int e = 0; e < 4; ++e) k4[e] = 0x7fff7fffu, v4[e] = 0;
        }
        if (!PLAIN) {
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
  auto store = [&](int t, int buf) {
    bool gone = false;
#pragma unroll
    for (int p = 0; p < NL; ++p) gone |= (sk[p] >> 16) != 0;
    if (t * KT + KT > hi_min || t * KT < lo_max || __ballot(gone) != 0) store_as(t, buf, std::false_type());
    else store_as(t, buf, std::true_type());
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
  // (the queries are here before the loop: in it, a wait for them would be one for every load)
#pragma unroll
  for (int j = 0; j < DP / 16; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      uint32_t x = qf[j][e];
      asm volatile("" : "+v"(x));
      qf[j][e] = x;
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
        if (tok >= hi || tok < lo) continue;
        const int c0 = fresh(4 * half);
#pragma unroll
        for (int c = 0; c < CB; ++c)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[c][i] += not_finite_value<FMT, T>(a, row, c0 + 32 * c + 8 * (i >> 2) + (i & 3));
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
      for (int i = 0; i < 16; i += 2) {
        const int ch = 32 * c + 8 * (i >> 2) + 4 * half + (i & 3);
        if (ch < D) store_coherent2(mine + ch, o[c][i], o[c][i + 1]);
      }
    if (half == 0) {
      qtea_detail::store_coherent(ml, m);
      qtea_detail::store_coherent(ml + kTaskRows, l);
    }
  }
  if (!last_to_arrive(a.counters + id * kCounterWords, used, &s_last)) return;
  // With up to 128 rows a thread has many items, so the parts' factors are
  // found once, in LDS, and two items' sums are asked for together (a
  // 200-token chunk in nine parts: 98 us, 110 with join_parts).
  float* s_f = reinterpret_cast<float*>(&s_k[0][0]);  // [rows][parts]: maxima, then factors
  float* s_w = s_f + kTaskRows * kMaxParts;           // sums
  static_assert(2 * kTaskRows * kMaxParts * 4 <= sizeof(s_k), "the parts' maxima and sums in LDS");
#pragma unroll 4
  for (int e = tid; e < kTaskRows * used; e += kThreads) {
    const int p = e / kTaskRows, row = min(e % kTaskRows, nrow - 1);
    const float* from = a.part_ml + (slot0 + p) * (2 * kTaskRows) + row;
    s_f[e % kTaskRows * kMaxParts + p] = qtea_detail::load_coherent(from);
    s_w[e % kTaskRows * kMaxParts + p] = qtea_detail::load_coherent(from + kTaskRows);
  }
  __syncthreads();
  if (tid < kTaskRows) {
    float* f = s_f + tid * kMaxParts;
    float* w = s_w + tid * kMaxParts;
    float M = -INFINITY, L = 0.0f;
    for (int p = 0; p < used; ++p) M = fmaxf(M, f[p]);
    for (int p = 0; p < used; ++p) {
      f[p] = f[p] == M ? 1.0f : __builtin_amdgcn_exp2f(f[p] - M);
      L += w[p] * f[p];
    }
    w[0] = L;
  }
  __syncthreads();
  const int quads = D / 4, items = nrow * quads;
  constexpr int kItems = 2, kBatch = 8;
  for (int e0 = tid; e0 < items; e0 += kItems * kThreads) {
    f32x4 acc[kItems];
    int row[kItems], ch[kItems];
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
      const int e = min(e0 + k * kThreads, items - 1);
      row[k] = e / quads, ch[k] = (e - row[k] * quads) * 4;
      acc[k] = f32x4{0, 0, 0, 0};
    }
    for (int p0 = 0; p0 < used; p0 += kBatch) {
      f32x2 x[kItems][kBatch], y[kItems][kBatch];
#pragma unroll
      for (int i = 0; i < kBatch; ++i)
#pragma unroll
        for (int k = 0; k < kItems; ++k) {
          const float* po = a.part + (slot0 + min(p0 + i, used - 1)) * (kTaskRows * DP) + row[k] * DP + ch[k];
          x[k][i] = load_coherent2(po), y[k][i] = load_coherent2(po + 2);
        }
#pragma unroll
      for (int i = 0; i < kBatch; ++i)
        if (p0 + i < used) {
#pragma unroll
          for (int k = 0; k < kItems; ++k) acc[k] += f32x4{x[k][i][0], x[k][i][1], y[k][i][0], y[k][i][1]} * s_f[row[k] * kMaxParts + p0 + i];
        }
    }
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
      if (e0 + k * kThreads >= items) continue;
      const int r = r0 + row[k], i = r / G;
      const float L = s_w[row[k] * kMaxParts], inv = pos0 + i < 0 && L == 0.0f ? 0.0f : 1.0f / L;
      uint16_t* to = a.out + (int64_t(q.first) + i) * a.out_stride + int64_t(h * G + (r - i * G)) * D + ch[k];
      *reinterpret_cast<u32x2*>(to) = u32x2{T::pack(acc[k][0] * inv, acc[k][1] * inv), T::pack(acc[k][2] * inv, acc[k][3] * inv)};
    }
  }
}

int device_cus() {
  static std::atomic<int> known[qtea_detail::kMaxDevices];
  return qtea_detail::per_current_device(known, [](int dev) {
    int n = 0;
    return hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) == hipSuccess ? n : 0;
  });
}

// The workspace: counters, the parts' maxima and sums, the parts.  The kernel
// for few rows has a slot for every chunk of a split task, of which there are
// no more than workgroups where all chunks fit them, and else less than
// 2 / 1.5 of that (a split task's last chunk is the only one that may be short).
constexpr int kRowsMax = 64;
constexpr int kSlotsPerCu = 5;
struct WsLayout {
  int64_t ml, part, bytes;
};
int padded_dim(int dim) { return dim <= 64 ? 64 : (dim <= 128 ? 128 : 256); }
WsLayout ws_layout(int dim, int cus) {
  static_assert(kSlotsPerCu * kRowsMax >= kWgPerCu * kTaskRows, "the other kernel's parts, one a workgroup");
  const int64_t rows = int64_t(cus) * kSlotsPerCu * kRowsMax;
  WsLayout w;
  w.ml = 2 * 4 * int64_t(cus) * kSlotsPerCu * kCounterWords;  // counters, maxima and sums: of two levels
  w.part = w.ml + rows * 2 * 2 * 4;
  w.bytes = w.part + rows * padded_dim(dim) * 4;
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
  const float scale_log2 = scale * 1.44269504088896341f;
  if (!(scale > 0.0f) || !std::isfinite(scale_log2) || window < 0) return QTEA_ERR_INVALID_ARG;
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
  a.scale = scale_log2;
  a.max_slots = cus * kSlotsPerCu;
  char* ws = static_cast<char*>(workspace);
  a.counters = reinterpret_cast<uint32_t*>(ws);
  a.part_ml = reinterpret_cast<float*>(ws + wl.ml);
  a.part = reinterpret_cast<float*>(ws + wl.part);
  const dim3 block(kThreads);
  const hipStream_t st = static_cast<hipStream_t>(stream);
  // The kernel by a sequence's rows on average (a call's lengths are only
  // known on the device; with more than a token each, some have more).
  const int64_t likely = batch->n_tokens > batch->n_seq ? rows + rows / 3 : rows;
  const int halves = likely <= int64_t(16) * batch->n_seq ? 1 : (likely <= int64_t(32) * batch->n_seq || D > 128 ? 2 : 4);
  const bool many = rows > int64_t(D > 128 ? 32 : 64) * batch->n_seq;
  const int64_t tasks = rows / kTaskRows + batch->n_seq, grid = int64_t(cus) * kWgPerCu;  // (tasks per head, at most)
  const int parts = int(std::max<int64_t>(1, std::min<int64_t>(grid / (tasks * H), kMaxParts)));
  if (many && tasks * H * parts > INT32_MAX) return QTEA_ERR_INVALID_ARG;
  auto launch = [&](auto dp, auto fmt, auto ty) {
    constexpr int DP = decltype(dp)::value, FMT = decltype(fmt)::value;
    using T = decltype(ty);
    if (many) {
      const dim3 wgs(uint32_t(tasks * H * parts));
      if (D == DP) hipLaunchKernelGGL((attn_tile_kernel<DP, FMT, T, true>), wgs, block, 0, st, a, parts);
      else hipLaunchKernelGGL((attn_tile_kernel<DP, FMT, T, false>), wgs, block, 0, st, a, parts);
      return;
    }
    auto rows_launch = [&](auto r) {
      constexpr int R = decltype(r)::value;
      const dim3 wgs(cus * rows_per_cu(DP, FMT, R)), threads(kRowThreads);
      if (D == DP) hipLaunchKernelGGL((attn_rows_kernel<DP, FMT, T, R, true>), wgs, threads, 0, st, a);
      else hipLaunchKernelGGL((attn_rows_kernel<DP, FMT, T, R, false>), wgs, threads, 0, st, a);
    };
    if (halves == 1) rows_launch(std::integral_constant<int, 1>());
    else if (halves == 2) rows_launch(std::integral_constant<int, 2>());
    else if constexpr (DP <= 128) rows_launch(std::integral_constant<int, 4>());
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
