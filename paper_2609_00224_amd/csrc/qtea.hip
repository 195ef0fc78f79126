// Compressed ternary GEMV for gfx950: packing, read-back, the streaming-read
// measurement kernel and their part of the C ABI declared in include/qtea.h
// (the GEMV kernels and entry points are in grouped.hip and grouped_mma.hip).
//
// Device layout (layout versions 2 and 3), all regions 256-byte aligned:
//   header   256 B: magic, layout, sizes; a validation flag word at +128.
//   trits    [n_pad/64 tiles][n_groups][64 rows][16 bytes]
//            One 16-byte unit holds the sixteen packs of one 16-pack group
//            for one row; a wavefront (64 lanes = 64 rows of a tile) reads
//            1 KiB contiguous per 128-bit load.  Byte i of the unit of row r
//            holds pack 16*g + ((i + r) mod 16): rows are rotated so that at
//            step i the 16 lanes of a quarter-wave address 16 different
//            packs' table columns (distinct LDS banks).
//   alpha    fp16 [n_pad]              (zero in the row padding)
//   v        fp16 [n_groups * 80]      (zero in the column padding)
//   salient  int32 [n_salient]
//   spos     int32 [n_groups + 1]      first s with S_s >= 80 * g
//   rval     [n_pad/64][n_salient][16] fp16 (layout 2) or FP8 E4M3 bytes
//            (layout 3): residual of four-row group g in salient
//            column s at ((g / 16) * n_salient + s) * 16 + g % 16: the sixteen
//            groups of a tile are contiguous per column, and a tile's residual
//            over a run of salient columns is one contiguous run
//   ridx     u32  [n_pad/64][n_salient] 2-bit positions of 16 consecutive groups
//
#include "qtea_internal.h"

namespace {

using namespace qtea_detail;


// ---------------------------------------------------------------------------
// Packing kernels (offline).
// ---------------------------------------------------------------------------
__global__ void validate_kernel(const int8_t* __restrict__ trits, int64_t nt,
                                const uint8_t* __restrict__ ridx, int64_t ni,
                                const int32_t* __restrict__ S, int64_t nS, int64_t K,
                                uint32_t* __restrict__ flags) {
  uint32_t f = 0;
  const int64_t stride = int64_t(gridDim.x) * blockDim.x;
  for (int64_t i = int64_t(blockIdx.x) * blockDim.x + threadIdx.x; i < nt; i += stride) {
    const int8_t t = trits[i];
    if (t < -1 || t > 1) f |= kFlagBadTrit;
  }
  for (int64_t i = int64_t(blockIdx.x) * blockDim.x + threadIdx.x; i < ni; i += stride)
    if (ridx[i] > 3) f |= kFlagBadResid;
  for (int64_t s = int64_t(blockIdx.x) * blockDim.x + threadIdx.x; s < nS; s += stride) {
    const int32_t c = S[s];
    if (c < 0 || c >= K || (s > 0 && c <= S[s - 1])) f |= kFlagBadResid;
  }
  if (f) atomicOr(flags, f);
}

// One thread per 16-byte unit (tile, group, row-in-tile).
__global__ void pack_trits_kernel(const int8_t* __restrict__ trits, int64_t N, int64_t K,
                                  int64_t n_groups, int64_t n_units, uint8_t* __restrict__ out) {
  const int64_t stride = int64_t(gridDim.x) * blockDim.x;
  for (int64_t u = int64_t(blockIdx.x) * blockDim.x + threadIdx.x; u < n_units; u += stride) {
    const int64_t l = u % kTileRows;
    const int64_t g = (u / kTileRows) % n_groups;
    const int64_t tile = u / (kTileRows * n_groups);
    const int64_t r = tile * kTileRows + l;
    uint32_t w[4] = {kZeroCode4, kZeroCode4, kZeroCode4, kZeroCode4};
    if (r < N) {
      const int8_t* row = trits + r * K;
      for (int i = 0; i < kGroupPacks; ++i) {
        const int64_t p = g * kGroupPacks + ((i + l) & (kGroupPacks - 1));
        uint32_t code = 0, pw = 1;
        for (int e = 0; e < 5; ++e) {
          const int64_t j = 5 * p + e;
          int t = j < K ? row[j] : 0;
          t = t < -1 ? -1 : (t > 1 ? 1 : t);  // invalid input is reported by validate_kernel
          code += uint32_t(t + 1) * pw;
          pw *= 3;
        }
        const int sh = 8 * (i & 3);
        w[i >> 2] = (w[i >> 2] & ~(0xffu << sh)) | (code << sh);
      }
    }
    const u32x4 v = {w[0], w[1], w[2], w[3]};
    *reinterpret_cast<u32x4*>(out + u * 16) = v;
  }
}

// Scales, salient list and residual blocks.  VT is the residual value type:
// uint16_t (fp16 bits, layout 2; an infinity or NaN is flagged) or uint8_t
// (E4M3 bytes, layout 3; a NaN code is flagged).  Finite values let the
// kernels pad a part's salient columns with duplicates whose products with
// a zero activation are exact zeros.  With S == o_S the salient list is already in place (derived
// from a bitmap) and only read.
template <typename VT>
__global__ void pack_meta_kernel(const uint16_t* __restrict__ alpha, const uint16_t* __restrict__ v,
                                 const int32_t* S, const VT* __restrict__ rval,
                                 const uint8_t* __restrict__ ridx, int64_t N, int64_t K, int64_t nS,
                                 int64_t n_pad, int64_t n_groups, uint16_t* __restrict__ o_alpha,
                                 uint16_t* __restrict__ o_v, int32_t* o_S,
                                 int32_t* __restrict__ o_spos, VT* __restrict__ o_rval,
                                 uint32_t* __restrict__ o_ridx, uint32_t* __restrict__ flags, int g128) {
  const int64_t stride = int64_t(gridDim.x) * blockDim.x;
  const int64_t t0 = int64_t(blockIdx.x) * blockDim.x + threadIdx.x;
  if (o_alpha)  // layout 4: scales and v by pack_scales128_kernel
    for (int64_t i = t0; i < n_pad; i += stride) o_alpha[i] = i < N ? alpha[i] : 0;
  if (o_v)
    for (int64_t i = t0; i < n_groups * kGroupCols; i += stride) o_v[i] = i < K ? v[i] : 0;
  if (S != o_S)
    for (int64_t i = t0; i < nS; i += stride) o_S[i] = S[i];
  for (int64_t g = t0; g <= n_groups; g += stride) {
    // lower bound of the first column of 16-pack group g in the sorted
    // salient list (layout 4: slot g holds columns from 128 (g / 2) + 65 (g % 2))
    int64_t lo = 0, hi = nS;
    const int64_t key = g128 ? g128_slot_col0(g) : g * kGroupCols;
    while (lo < hi) {
      const int64_t mid = (lo + hi) / 2;
      if (S[mid] < key)
        lo = mid + 1;
      else
        hi = mid;
    }
    o_spos[g] = int32_t(lo);
  }
  const int64_t G = N / 4, Gp = n_pad / 4, Wp = n_pad / 64;
  uint32_t f = 0;
  for (int64_t i = t0; i < nS * Gp; i += stride) {
    const int64_t tile = i / (16 * nS), rem = i - tile * 16 * nS;
    const int64_t s = rem >> 4, g = 16 * tile + (rem & 15);
    const VT val = g < G ? rval[s * G + g] : VT(0);
    if (sizeof(VT) == 1 ? e4m3_is_nan(uint8_t(val)) : (uint32_t(val) & 0x7c00u) == 0x7c00u) f |= kFlagBadResid;
    o_rval[i] = val;
  }
  if (f) atomicOr(flags, f);
  for (int64_t i = t0; i < nS * Wp; i += stride) {
    const int64_t w = i / nS, s = i % nS;
    uint32_t word = 0;
    for (int k = 0; k < 16; ++k) {
      const int64_t g = 16 * w + k;
      if (g < G) word |= uint32_t(ridx[s * G + g] & 3) << (2 * k);
    }
    o_ridx[i] = word;
  }
}

// Salient column list from a column bitmap (bit j % 32 of word j / 32 set
// when column j is salient), ascending, by one workgroup: each thread counts
// a contiguous run of words, a scan over the threads gives every run's first
// list position.  A bit at or past K, or a count other than nS, is flagged
// (and nothing is written).
__global__ __launch_bounds__(1024) void bitmap_salient_kernel(const uint32_t* __restrict__ bitmap,
                                                              int64_t K, int64_t nS,
                                                              int32_t* __restrict__ o_S,
                                                              uint32_t* __restrict__ flags) {
  __shared__ int64_t run[1024];
  const int t = threadIdx.x;
  const int64_t nw = (K + 31) / 32, per = (nw + 1023) / 1024;
  const int64_t w0 = min(nw, int64_t(t) * per), w1 = min(nw, w0 + per);
  const uint32_t tail = (K & 31) ? (1u << (K & 31)) - 1u : 0xffffffffu;
  uint32_t f = 0;
  int64_t cnt = 0;
  for (int64_t w = w0; w < w1; ++w) {
    uint32_t b = bitmap[w];
    if (w == nw - 1) {
      if (b & ~tail) f |= kFlagBadResid;
      b &= tail;
    }
    cnt += __popc(b);
  }
  run[t] = cnt;
  __syncthreads();
  for (int off = 1; off < 1024; off <<= 1) {  // inclusive scan
    const int64_t add = t >= off ? run[t - off] : 0;
    __syncthreads();
    run[t] += add;
    __syncthreads();
  }
  if (run[1023] != nS) {
    f |= kFlagBadResid;
  } else {
    int64_t pos = run[t] - cnt;
    for (int64_t w = w0; w < w1; ++w) {
      uint32_t b = bitmap[w] & (w == nw - 1 ? tail : 0xffffffffu);
      while (b) {
        o_S[pos++] = int32_t(32 * w + (__ffs(b) - 1));
        b &= b - 1u;
      }
    }
  }
  if (f) atomicOr(flags, f);
}

__global__ void write_header_kernel(uint8_t* packed, int64_t N, int64_t K, int64_t nS, int layout) {
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    uint32_t* h = reinterpret_cast<uint32_t*>(packed);
    h[0] = QTEA_DESC_MAGIC;
    h[1] = uint32_t(layout);
    int64_t* h64 = reinterpret_cast<int64_t*>(packed + 8);
    h64[0] = N;
    h64[1] = K;
    h64[2] = nS;
    reinterpret_cast<uint32_t*>(packed + kFlagOffset)[0] = 0;
  }
}

// Layout 4 trits: one thread per 13-byte row of a slot (tile, 16-pack slot
// dg, row l), at byte 13 ((tile n_groups + dg) 64 + l).  Byte i holds pack
// (i + (l mod 16)) mod 13 of the slot, i.e. pack 13 (dg % 2) + that of
// quantization group dg / 2, which codes the group's columns 5p..5p+4 (zero
// trits past its column 127 and past K).  The rotation by the row spreads
// the rows of a wave's lookups over the table's columns.
__global__ void pack_trits128_kernel(const int8_t* __restrict__ trits, int64_t N, int64_t K,
                                     int64_t n_groups, int64_t n_units, uint8_t* __restrict__ out) {
  const int64_t stride = int64_t(gridDim.x) * blockDim.x;
  for (int64_t u = int64_t(blockIdx.x) * blockDim.x + threadIdx.x; u < n_units; u += stride) {
    const int64_t l = u % kTileRows;
    const int64_t dg = (u / kTileRows) % n_groups;
    const int64_t tile = u / (kTileRows * n_groups);
    const int64_t r = tile * kTileRows + l, g = dg >> 1;
    uint8_t* dst = out + u * kG128SlotPacks;
    for (int i = 0; i < kG128SlotPacks; ++i) {
      const int64_t p = kG128SlotPacks * (dg & 1) + (i + (l & 15)) % kG128SlotPacks;
      uint32_t code = 0, pw = 1;
      for (int e = 0; e < 5; ++e) {
        const int64_t c = 5 * p + e, j = kScaleCols * g + c;
        int t = (r < N && c < kScaleCols && j < K) ? trits[r * K + j] : 0;
        t = t < -1 ? -1 : (t > 1 ? 1 : t);  // invalid input is reported by validate_kernel
        code += uint32_t(t + 1) * pw;
        pw *= 3;
      }
      dst[i] = uint8_t(code);
    }
  }
}

// Layout 4 scales and rescales: (alpha | beta << 16) per row and group as
// [n_pad/64][n_sg][64] (zero in padded rows), v in device column order
// (device column c < 65 of slot dg is the group's column 65 (dg % 2) + c;
// zero past it).
__global__ void pack_scales128_kernel(const uint16_t* __restrict__ alpha, const uint16_t* __restrict__ beta,
                                      const uint16_t* __restrict__ v, int64_t N, int64_t K, int64_t n_pad,
                                      int64_t n_sg, uint32_t* __restrict__ o_ab, uint16_t* __restrict__ o_v) {
  const int64_t stride = int64_t(gridDim.x) * blockDim.x;
  const int64_t t0 = int64_t(blockIdx.x) * blockDim.x + threadIdx.x;
  for (int64_t i = t0; i < n_pad * n_sg; i += stride) {
    const int64_t tile = i / (n_sg * kTileRows), rem = i - tile * n_sg * kTileRows;
    const int64_t g = rem / kTileRows, r = tile * kTileRows + rem % kTileRows;
    o_ab[i] = r < N ? uint32_t(alpha[r * n_sg + g]) | (uint32_t(beta[r * n_sg + g]) << 16) : 0u;
  }
  for (int64_t i = t0; i < 2 * n_sg * kGroupCols; i += stride) {
    const int64_t dg = i / kGroupCols, col = i % kGroupCols;
    const int64_t c = kG128SlotCols * (dg & 1) + col, j = kScaleCols * (dg >> 1) + c;
    o_v[i] = (col < kG128SlotCols && c < kScaleCols && j < K) ? v[j] : uint16_t(0);
  }
}

// The vs region (u32 per device column): pass 1 copies the v bits, pass 2
// marks every salient column with 1 + its rank among the salient columns of
// its 320-column slice (device columns; layout 4 maps column j to device
// column g128_dcol(j)).
__global__ void pack_vs_kernel(const uint16_t* __restrict__ o_v, int64_t n_cols, uint32_t* __restrict__ o_vs) {
  const int64_t stride = int64_t(gridDim.x) * blockDim.x;
  for (int64_t i = int64_t(blockIdx.x) * blockDim.x + threadIdx.x; i < n_cols; i += stride) o_vs[i] = o_v[i];
}
// A salient list that failed validation (reported by the pack's flags) may
// hold any value: every index is checked before it is used.
__global__ void mark_salient_kernel(const int32_t* __restrict__ S, const int32_t* __restrict__ spos, int64_t nS,
                                    int64_t K, int64_t n_groups, int g128, uint32_t* __restrict__ o_vs) {
  const int64_t stride = int64_t(gridDim.x) * blockDim.x;
  for (int64_t s = int64_t(blockIdx.x) * blockDim.x + threadIdx.x; s < nS; s += stride) {
    const int64_t j = S[s];
    if (j < 0 || j >= K) continue;
    const int64_t dc = g128 ? g128_dcol(j) : j;
    const int64_t g0 = 4 * (dc / (4 * kGroupCols));
    if (dc >= n_groups * kGroupCols || g0 > n_groups) continue;
    const int64_t rank = s - spos[g0];
    if (rank < 0 || rank >= 4 * kGroupCols) continue;
    o_vs[dc] |= uint32_t(rank + 1) << 16;
  }
}

// Streaming-read ceiling: each workgroup of 256 streams one contiguous 64 KiB
// chunk with 16-byte non-temporal loads, eight in flight per thread (under
// sustained load this holds about 7 TB/s, grid-stride loads about 6.5), and
// stores the fold of its chunk to its own word of sink: one atomic per
// workgroup on a shared word instead would cost more than a third of the rate.
constexpr int kCeilUnroll = 8;
constexpr int kCeilThreads = 256;
constexpr int64_t kCeilChunk16 = int64_t(QTEA_READ_CEILING_CHUNK) / 16;
// (The chunk length is a kernel argument: the loop's code is then the one
// measured at the rate above.)
__global__ __launch_bounds__(kCeilThreads) void read_ceiling_kernel(const u32x4* __restrict__ buf, int64_t n16,
                                                                    int64_t chunk16, uint32_t* __restrict__ sink) {
  const int64_t b0 = int64_t(blockIdx.x) * chunk16;
  const int64_t b1 = b0 + chunk16 < n16 ? b0 + chunk16 : n16;
  uint32_t f = 0;
  int64_t i = b0 + threadIdx.x;
  for (; i + (kCeilUnroll - 1) * kCeilThreads < b1; i += kCeilUnroll * kCeilThreads) {
    u32x4 v[kCeilUnroll];
#pragma unroll
    for (int k = 0; k < kCeilUnroll; ++k) v[k] = __builtin_nontemporal_load(buf + i + k * kCeilThreads);
#pragma unroll
    for (int k = 0; k < kCeilUnroll; ++k) f ^= v[k].x + v[k].y + v[k].z + v[k].w;
  }
  for (; i < b1; i += kCeilThreads) {
    const u32x4 a = __builtin_nontemporal_load(buf + i);
    f ^= a.x + a.y + a.z + a.w;
  }
  for (int o = 32; o > 0; o >>= 1) f ^= __shfl_xor(f, o);
  __shared__ uint32_t red[kCeilThreads / 64];
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = f;
  __syncthreads();
  if (threadIdx.x == 0) {
    uint32_t t = 0;
    for (int k = 0; k < kCeilThreads / 64; ++k) t ^= red[k];
    sink[blockIdx.x] = t;
  }
}

// ---------------------------------------------------------------------------
// Debug unpack (bit-exact read-back of the layout).
// ---------------------------------------------------------------------------
__global__ void unpack_codes_kernel(const uint8_t* __restrict__ tr, int64_t N, int64_t K,
                                    int64_t n_packs, int64_t n_groups, uint8_t* __restrict__ canon,
                                    int8_t* __restrict__ trits) {
  const int64_t stride = int64_t(gridDim.x) * blockDim.x;
  for (int64_t e = int64_t(blockIdx.x) * blockDim.x + threadIdx.x; e < N * n_packs; e += stride) {
    const int64_t r = e / n_packs, p = e % n_packs;
    const int64_t tile = r / kTileRows, l = r % kTileRows;
    const int64_t g = p / kGroupPacks, q = p % kGroupPacks;
    const int64_t i = (q - l) & (kGroupPacks - 1);
    const uint8_t c = tr[((tile * n_groups + g) * kTileRows + l) * 16 + i];
    if (canon) canon[e] = c;
    if (trits) {
      uint32_t rest = c;
      for (int d = 0; d < 5; ++d) {
        const int64_t j = 5 * p + d;
        if (j < K) trits[r * K + j] = int8_t(int(rest % 3) - 1);
        rest /= 3;
      }
    }
  }
}

// Layout 4: the paper's codes [N][26 n_sg] (26 per row and group) and trits.
__global__ void unpack_codes128_kernel(const uint8_t* __restrict__ tr, int64_t N, int64_t K,
                                       int64_t n_packs, int64_t n_groups, uint8_t* __restrict__ canon,
                                       int8_t* __restrict__ trits) {
  const int64_t stride = int64_t(gridDim.x) * blockDim.x;
  for (int64_t e = int64_t(blockIdx.x) * blockDim.x + threadIdx.x; e < N * n_packs; e += stride) {
    const int64_t r = e / n_packs, pp = e % n_packs;
    const int64_t g = pp / kScalePacks, p = pp % kScalePacks;
    const int64_t tile = r / kTileRows, l = r % kTileRows, dg = 2 * g + p / kG128SlotPacks;
    const int64_t i = ((p % kG128SlotPacks) - (l & 15) + 2 * kG128SlotPacks) % kG128SlotPacks;
    const uint8_t c = tr[((tile * n_groups + dg) * kTileRows + l) * kG128SlotPacks + i];
    if (canon) canon[e] = c;
    if (trits) {
      uint32_t rest = c;
      for (int d = 0; d < 5; ++d) {
        const int64_t col = 5 * p + d, j = kScaleCols * g + col;
        if (col < kScaleCols && j < K) trits[r * K + j] = int8_t(int(rest % 3) - 1);
        rest /= 3;
      }
    }
  }
}

__global__ void unpack_resid_kernel(const uint32_t* __restrict__ ridx, int64_t N, int64_t nS,
                                    int64_t n_pad, int32_t* __restrict__ rows) {
  const int64_t G = N / 4;
  const int64_t stride = int64_t(gridDim.x) * blockDim.x;
  for (int64_t e = int64_t(blockIdx.x) * blockDim.x + threadIdx.x; e < nS * G; e += stride) {
    const int64_t s = e / G, g = e % G;
    const uint32_t w = ridx[(g / 16) * nS + s];
    rows[e] = int32_t(4 * g + ((w >> (2 * (g % 16))) & 3));
  }
}

__global__ void fill_zero_kernel(uint32_t* __restrict__ p, int64_t n_words, uint8_t* __restrict__ tail,
                                 int64_t n_tail) {
  const int64_t stride = int64_t(gridDim.x) * blockDim.x;
  const int64_t t0 = int64_t(blockIdx.x) * blockDim.x + threadIdx.x;
  for (int64_t i = t0; i < n_words; i += stride) p[i] = 0;
  for (int64_t i = t0; i < n_tail; i += stride) tail[i] = 0;
}

int grid_for(int64_t n, int64_t per_thread_block = 256) {
  int64_t g = cdiv(n, per_thread_block);
  if (g < 1) g = 1;
  if (g > 65536) g = 65536;
  return int(g);
}

}  // namespace

// ---------------------------------------------------------------------------
// C ABI.
// ---------------------------------------------------------------------------
extern "C" {

const char* qtea_status_string(int status) {
  switch (status) {
    case QTEA_OK: return "ok";
    case QTEA_ERR_INVALID_ARG: return "invalid argument";
    case QTEA_ERR_BAD_TRIT: return "trit outside {-1, 0, +1}";
    case QTEA_ERR_BAD_RESIDUAL: return "bad residual position or salient column list";
    case QTEA_ERR_BATCH: return "batch outside [1, 16] (4-bit weights: [1, 64])";
    case QTEA_ERR_WORKSPACE: return "workspace or packed buffer too small";
    case QTEA_ERR_HIP: return "HIP runtime error";
    case QTEA_ERR_NOT_POSITIVE: return "Hessian not positive definite";
    default: return "unknown status";
  }
}

int qtea_abi_version(void) { return QTEA_ABI_VERSION; }

int qtea_packed_bytes(int64_t N, int64_t K, int64_t n_salient, int64_t* out_bytes) {
  Layout L;
  if (!out_bytes || !make_layout(N, K, n_salient, &L)) return QTEA_ERR_INVALID_ARG;
  *out_bytes = L.total;
  return QTEA_OK;
}

int qtea_packed_bytes_e4m3(int64_t N, int64_t K, int64_t n_salient, int64_t* out_bytes) {
  Layout L;
  if (!out_bytes || !make_layout(N, K, n_salient, &L, kLayoutE4M3)) return QTEA_ERR_INVALID_ARG;
  *out_bytes = L.total;
  return QTEA_OK;
}

}  // extern "C"

namespace {

// The pack entry points: layout 2 takes a salient list and fp16 residual
// values, layout 3 a salient bitmap and E4M3 residual bytes, layout 4 that
// and per-row, per-128-column-group scales and biases (row_scale and
// row_bias [N][ceil(K/128)]).
int pack_any(int layout, const int8_t* trits, int64_t N, int64_t K, const uint16_t* row_scale,
             const uint16_t* row_bias, const uint16_t* col_rescale, const int32_t* salient,
             const uint32_t* bitmap, int64_t n_salient, const void* resid_val, const uint8_t* resid_idx,
             void* packed, int64_t packed_bytes, qtea_desc* out_desc, void* stream) {
  Layout L;
  if (!out_desc) return QTEA_ERR_INVALID_ARG;
  out_desc->magic = 0;
  if (!make_layout(N, K, n_salient, &L, layout)) return QTEA_ERR_INVALID_ARG;
  if (!trits || !row_scale || !col_rescale || !packed) return QTEA_ERR_INVALID_ARG;
  if (layout == kLayoutG128 && !row_bias) return QTEA_ERR_INVALID_ARG;
  if (n_salient > 0 && (!resid_val || !resid_idx)) return QTEA_ERR_INVALID_ARG;
  if (layout == kLayout ? (n_salient > 0 && !salient) : !bitmap) return QTEA_ERR_INVALID_ARG;
  if (packed_bytes < L.total) return QTEA_ERR_WORKSPACE;
  hipStream_t st = static_cast<hipStream_t>(stream);
  uint8_t* pk = static_cast<uint8_t*>(packed);
  uint32_t* flags = reinterpret_cast<uint32_t*>(pk + kFlagOffset);
  int32_t* o_S = reinterpret_cast<int32_t*>(pk + L.off_salient);

  hipLaunchKernelGGL(write_header_kernel, dim3(1), dim3(64), 0, st, pk, N, K, n_salient, layout);
  const int64_t ni = n_salient * (N / 4);
  // the salient list given is checked here; one derived from a bitmap is
  // checked as it is derived
  hipLaunchKernelGGL(validate_kernel, dim3(grid_for(N * K, 256 * 16)), dim3(256), 0, st, trits, N * K,
                     resid_idx, ni, layout == kLayout ? salient : nullptr,
                     layout == kLayout ? n_salient : int64_t(0), K, flags);
  if (layout != kLayout) {
    hipLaunchKernelGGL(bitmap_salient_kernel, dim3(1), dim3(1024), 0, st, bitmap, K, n_salient, o_S, flags);
    salient = o_S;
  }
  const int64_t n_units = L.n_tiles * L.n_groups * kTileRows;
  if (layout == kLayoutG128) {
    const int64_t n_sg = L.n_groups / 2;
    hipLaunchKernelGGL(pack_trits128_kernel, dim3(grid_for(n_units)), dim3(256), 0, st, trits, N, K,
                       L.n_groups, n_units, pk + L.off_trits);
    hipLaunchKernelGGL(pack_scales128_kernel, dim3(grid_for(L.n_pad * n_sg)), dim3(256), 0, st, row_scale,
                       row_bias, col_rescale, N, K, L.n_pad, n_sg, reinterpret_cast<uint32_t*>(pk + L.off_alpha),
                       reinterpret_cast<uint16_t*>(pk + L.off_v));
  } else {
    hipLaunchKernelGGL(pack_trits_kernel, dim3(grid_for(n_units)), dim3(256), 0, st, trits, N, K,
                       L.n_groups, n_units, pk + L.off_trits);
  }
  const int64_t meta_n = L.n_pad + L.n_groups * kGroupCols + n_salient * (L.n_pad / 4);
  uint16_t* o_alpha = layout == kLayoutG128 ? nullptr : reinterpret_cast<uint16_t*>(pk + L.off_alpha);
  uint16_t* o_v = layout == kLayoutG128 ? nullptr : reinterpret_cast<uint16_t*>(pk + L.off_v);
  int32_t* o_spos = reinterpret_cast<int32_t*>(pk + L.off_spos);
  uint32_t* o_ridx = reinterpret_cast<uint32_t*>(pk + L.off_ridx);
  if (layout == kLayout)
    hipLaunchKernelGGL(pack_meta_kernel<uint16_t>, dim3(grid_for(meta_n)), dim3(256), 0, st, row_scale,
                       col_rescale, salient, static_cast<const uint16_t*>(resid_val), resid_idx, N, K,
                       n_salient, L.n_pad, L.n_groups, o_alpha, o_v, o_S, o_spos,
                       reinterpret_cast<uint16_t*>(pk + L.off_rval), o_ridx, flags, 0);
  else
    hipLaunchKernelGGL(pack_meta_kernel<uint8_t>, dim3(grid_for(meta_n)), dim3(256), 0, st, row_scale,
                       col_rescale, salient, static_cast<const uint8_t*>(resid_val), resid_idx, N, K,
                       n_salient, L.n_pad, L.n_groups, o_alpha, o_v, o_S, o_spos, pk + L.off_rval, o_ridx,
                       flags, int(layout == kLayoutG128));
  {
    uint32_t* o_vs = reinterpret_cast<uint32_t*>(pk + L.off_vs);
    const uint16_t* v_dev = reinterpret_cast<const uint16_t*>(pk + L.off_v);
    const int64_t n_cols = L.n_groups * kGroupCols;
    hipLaunchKernelGGL(pack_vs_kernel, dim3(grid_for(n_cols)), dim3(256), 0, st, v_dev, n_cols, o_vs);
    if (n_salient > 0)
      hipLaunchKernelGGL(mark_salient_kernel, dim3(grid_for(n_salient)), dim3(256), 0, st, o_S, o_spos, n_salient,
                         K, L.n_groups, int(layout == kLayoutG128), o_vs);
  }
  if (hipGetLastError() != hipSuccess) return QTEA_ERR_HIP;
  uint32_t hflags = 0;
  if (hipMemcpyAsync(&hflags, flags, 4, hipMemcpyDeviceToHost, st) != hipSuccess) return QTEA_ERR_HIP;
  if (hipStreamSynchronize(st) != hipSuccess) return QTEA_ERR_HIP;
  if (hflags & kFlagBadTrit) return QTEA_ERR_BAD_TRIT;
  if (hflags & kFlagBadResid) return QTEA_ERR_BAD_RESIDUAL;

  const qtea_desc d = desc_from_layout(L, N, K, n_salient, layout);
  *out_desc = d;
  return QTEA_OK;
}

}  // namespace

extern "C" {

int qtea_pack(const int8_t* trits, int64_t N, int64_t K, const uint16_t* row_scale,
              const uint16_t* col_rescale, const int32_t* salient, int64_t n_salient,
              const uint16_t* resid_val, const uint8_t* resid_idx, void* packed,
              int64_t packed_bytes, qtea_desc* out_desc, void* stream) {
  return pack_any(kLayout, trits, N, K, row_scale, nullptr, col_rescale, salient, nullptr, n_salient, resid_val,
                  resid_idx, packed, packed_bytes, out_desc, stream);
}

int qtea_pack_e4m3(const int8_t* trits, int64_t N, int64_t K, const uint16_t* row_scale,
                   const uint16_t* col_rescale, const uint32_t* salient_bitmap, int64_t n_salient,
                   const uint8_t* resid_val, const uint8_t* resid_idx, void* packed, int64_t packed_bytes,
                   qtea_desc* out_desc, void* stream) {
  return pack_any(kLayoutE4M3, trits, N, K, row_scale, nullptr, col_rescale, nullptr, salient_bitmap, n_salient,
                  resid_val, resid_idx, packed, packed_bytes, out_desc, stream);
}

int qtea_packed_bytes_g128(int64_t N, int64_t K, int64_t n_salient, int64_t* out_bytes) {
  Layout L;
  if (!out_bytes || !make_layout(N, K, n_salient, &L, kLayoutG128)) return QTEA_ERR_INVALID_ARG;
  *out_bytes = L.total;
  return QTEA_OK;
}

int qtea_pack_g128(const int8_t* trits, int64_t N, int64_t K, const uint16_t* group_scale,
                   const uint16_t* group_bias, const uint16_t* col_rescale, const uint32_t* salient_bitmap,
                   int64_t n_salient, const uint8_t* resid_val, const uint8_t* resid_idx, void* packed,
                   int64_t packed_bytes, qtea_desc* out_desc, void* stream) {
  return pack_any(kLayoutG128, trits, N, K, group_scale, group_bias, col_rescale, nullptr, salient_bitmap,
                  n_salient, resid_val, resid_idx, packed, packed_bytes, out_desc, stream);
}

int qtea_workspace_init(void* workspace, int64_t bytes, void* stream) {
  if (!workspace || bytes < 0 || (reinterpret_cast<uintptr_t>(workspace) & 3)) return QTEA_ERR_INVALID_ARG;
  if (bytes == 0) return QTEA_OK;
  const int64_t words = bytes / 4;
  hipLaunchKernelGGL(fill_zero_kernel, dim3(grid_for(words)), dim3(256), 0,
                     static_cast<hipStream_t>(stream), static_cast<uint32_t*>(workspace), words,
                     static_cast<uint8_t*>(workspace) + 4 * words, bytes - 4 * words);
  return hipGetLastError() == hipSuccess ? QTEA_OK : QTEA_ERR_HIP;
}

int qtea_read_ceiling(const void* buf, int64_t bytes, uint32_t* sink, void* stream) {
  if (!buf || !sink || bytes <= 0 || bytes % 16 != 0 || (reinterpret_cast<uintptr_t>(buf) & 15))
    return QTEA_ERR_INVALID_ARG;
  const int64_t n16 = bytes / 16, grid = (n16 + kCeilChunk16 - 1) / kCeilChunk16;
  if (grid > int64_t(INT32_MAX)) return QTEA_ERR_INVALID_ARG;
  hipLaunchKernelGGL(read_ceiling_kernel, dim3(uint32_t(grid)), dim3(kCeilThreads), 0,
                     static_cast<hipStream_t>(stream), static_cast<const u32x4*>(buf), n16, kCeilChunk16, sink);
  return hipGetLastError() == hipSuccess ? QTEA_OK : QTEA_ERR_HIP;
}

int qtea_debug_unpack(const qtea_desc* desc, const void* packed, uint8_t* canon_codes, int8_t* trits,
                      int32_t* resid_row, void* stream) {
  if (!desc_ok(desc) || !packed) return QTEA_ERR_INVALID_ARG;
  const qtea_desc& d = *desc;
  const uint8_t* pk = static_cast<const uint8_t*>(packed);
  hipStream_t st = static_cast<hipStream_t>(stream);
  if ((canon_codes || trits) && d.layout == kLayoutG128)
    hipLaunchKernelGGL(unpack_codes128_kernel, dim3(grid_for(d.N * d.n_packs)), dim3(256), 0, st,
                       pk + d.off_trits, d.N, d.K, d.n_packs, d.n_groups, canon_codes, trits);
  else if (canon_codes || trits)
    hipLaunchKernelGGL(unpack_codes_kernel, dim3(grid_for(d.N * d.n_packs)), dim3(256), 0, st,
                       pk + d.off_trits, d.N, d.K, d.n_packs, d.n_groups, canon_codes, trits);
  if (resid_row && d.n_salient > 0)
    hipLaunchKernelGGL(unpack_resid_kernel, dim3(grid_for(d.n_salient * (d.N / 4))), dim3(256), 0, st,
                       reinterpret_cast<const uint32_t*>(pk + d.off_ridx), d.N, d.n_salient, d.n_pad,
                       resid_row);
  return hipGetLastError() == hipSuccess ? QTEA_OK : QTEA_ERR_HIP;
}

}  // extern "C"
