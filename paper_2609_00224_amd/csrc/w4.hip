// Products of a few rows with a matrix of 4-bit codes.
//
// W [N][K] is packed in tiles of 16 rows by 128 columns, the left operand of four
// matrix instructions: lane (q, r) = 16 q + r of a wave holds row r, columns
// 32 q .. 32 q + 31, a block, as 16 bytes (code j in half j % 2 of byte j / 2).
//   codes   [ceil(K/128)][ceil(N/16)][64 lanes][16 bytes]
//   scales  [ceil(K/512)][ceil(N/16)][64 lanes][4 bytes], byte i that of tile 4 u + i
// Strips of 16 rows lie next to each other, so that what the waves of the chip
// read at a time, a column of tiles, is one piece (against strip after strip:
// 128257 x 4096 at 16 rows 50.0 us for 55.6, at one 49.4 for 53.0, both with loads
// that the caches keep).
// Rows and columns past the matrix are zeros.
#include <algorithm>
#include <type_traits>

#include "rows.h"

namespace qtea_serve {
namespace {

constexpr int kThreads = 512, kWaves = kThreads / 64;
constexpr int kTile = 1024;       // bytes of a tile's codes
constexpr int kUnitScales = 256;  // bytes of four tiles' scales
constexpr int kWideStrips = 4;    // strips of a wave where there are many

struct Layout {
  int64_t strips, tiles, units, scales_at, bytes;  // of 16 rows; tiles and units of four tiles of a strip
};
bool make_layout(int64_t N, int64_t K, Layout* l) {
  if (N < 1 || K < 1 || N > QTEA_W4_MAX_ROWS || K > (1 << 24)) return false;
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
  int64_t strips, tiles, units, total;  // total: strips * units * 256 blocks
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

// Done once for a matrix: 128257 x 4096 of fp16 350 us (1.33 GB, 3.8 TB/s), back 390.
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
      *reinterpret_cast<u32x4*>(a.codes + (k.tile * a.strips + k.strip) * kTile + k.lane * 16) = v;
    }
    a.scales[((k.tile >> 2) * a.strips + k.strip) * kUnitScales + k.lane * 4 + (k.tile & 3)] = uint8_t(e);
  }
}

template <int TYPE>
__global__ __launch_bounds__(kThreads) void w4_unpack_kernel(const PackArgs a) {
  for (int64_t b = int64_t(blockIdx.x) * kThreads + threadIdx.x; b < a.total; b += int64_t(gridDim.x) * kThreads) {
    const Block k = block_of(a, b);
    const int64_t row = k.strip * 16 + (k.lane & 15), col = k.tile * 128 + (k.lane >> 4) * 32;
    if (k.tile >= a.tiles || row >= a.N) continue;
    const float s = scale_value(a.scales[((k.tile >> 2) * a.strips + k.strip) * kUnitScales + k.lane * 4 + (k.tile & 3)]);
    const u32x4 v = *reinterpret_cast<const u32x4*>(a.codes + (k.tile * a.strips + k.strip) * kTile + k.lane * 16);
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
  int32_t x_bytes, x_scale_bytes;              // of X and its scales, first row to last
  int32_t N, K, strips, tiles, units, batch, y_type;
  bool x_dwords, y_wide;      // rows of X are 4-byte aligned, of Y (16 bits) 8-byte
  int32_t parts;              // waves that share a strip's units
};

// The 16-bit type whose matrix instructions a product runs on.  E4M3 activations
// become bf16 values, exactly: the instruction that takes 8-bit operands with
// their scales drops what lies 2^-16 below the largest of its products (measured).
template <int XT>
using Type = std::conditional_t<XT == QTEA_F16, F16, BF16>;

// 8 columns of the lane's block as the left operand: exact in either type.
template <class T>
__device__ __forceinline__ u32x4 weights(uint32_t w, float s) {
  return u32x4{T::template e2m1<0>(w, s), T::template e2m1<1>(w, s), T::template e2m1<2>(w, s), T::template e2m1<3>(w, s)};
}

typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));

// A lane's four rows n0.. of one result column (a row of Y).
__device__ __forceinline__ void store_y(const GemmArgs& a, int b, int64_t n0, f32x4 c) {
  if (b >= a.batch || n0 >= a.N) return;
  char* row = a.y + b * a.y_stride;
  const int size = a.y_type == QTEA_F32 ? 4 : 2;
  if (a.y_type == QTEA_F32 && n0 + 4 <= a.N) {
    *reinterpret_cast<f32x4u*>(row + 4 * n0) = c;
    return;
  }
  const u32x2 v = a.y_type == QTEA_F16 ? u32x2{F16::pack(c[0], c[1]), F16::pack(c[2], c[3])} : u32x2{BF16::pack(c[0], c[1]), BF16::pack(c[2], c[3])};
  if (a.y_wide && n0 + 4 <= a.N) {
    *reinterpret_cast<u32x2*>(row + 2 * n0) = v;
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (n0 + i >= a.N) break;
    if (size == 4) *reinterpret_cast<float*>(row + 4 * (n0 + i)) = c[i];
    else *reinterpret_cast<uint16_t*>(row + 2 * (n0 + i)) = uint16_t(v[i / 2] >> (16 * (i & 1)));
  }
}

// A strip's tile and scales from an address that is the same for the wave, which
// the compiler is to keep in scalar registers (and add the lanes' parts in the
// load, where it would carry 64-bit addresses a lane).
template <class V>
using global_t = __attribute__((address_space(1))) const V;
__device__ __forceinline__ uint64_t scalar(const uint8_t* p) {
  uint64_t at = reinterpret_cast<uint64_t>(p);
  asm volatile("" : "+s"(at));
  return at;
}
template <bool STREAM>
__device__ __forceinline__ u32x4 load_codes(uint64_t p, uint32_t lane, int r) {
  global_t<u32x4>* at = reinterpret_cast<global_t<u32x4>*>(p + lane * 16 + r * kTile);
  return STREAM ? __builtin_nontemporal_load(at) : *at;
}
__device__ __forceinline__ uint32_t load_scale4(uint64_t p, uint32_t lane, int r) { return *reinterpret_cast<global_t<uint32_t>*>(p + lane * 4 + r * kUnitScales); }

// A value that is computed where it is used instead of being held in
// registers across the loop.
__device__ __forceinline__ int fresh(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// X and its scales by way of descriptors: offsets past the end give zeros
// without a fetch, and 16-byte loads are aligned to 4 bytes.
struct XBuf {
  __amdgpu_buffer_rsrc_t x, scale;
};
template <int XT>
__device__ __forceinline__ XBuf x_buffers(const GemmArgs& a) {
  XBuf b;
  b.x = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(a.x), 0, a.x_bytes, 0x00020000);
  if constexpr (XT == QTEA_E4M3) b.scale = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(a.x_scale), 0, a.x_scale_bytes, 0x00020000);
  return b;
}

// 8 activations k.. of a row: 16-bit values, or codes and their block's scale.
// Zeros past K.
template <int XT>
struct Piece {
  std::conditional_t<XT == QTEA_E4M3, u32x2, u32x4> v;
  uint32_t scale;
};
constexpr uint32_t kPastEnd = 0x80000000u;  // an offset past every descriptor's end
// (Every lane of a wave takes part, whatever it needs: a number of loads that does
// not depend on the call lets the wave wait for the one it needs.)  ODD: rows
// that are 2-byte aligned.
template <int XT, bool ODD>
__device__ __forceinline__ Piece<XT> load_piece(const GemmArgs& a, const XBuf& xb, int row, int k) {
  Piece<XT> r;
  // (a row past the batch: a scalar offset past the end would not be the
  // descriptor's to refuse)
  const bool row_in = row < a.batch, in = row_in && k < a.K;
  const uint32_t at = in ? uint32_t(k) * elem_bytes(XT) : kPastEnd, row_at = row_in ? uint32_t(row) * uint32_t(a.x_stride) : 0u;
  if constexpr (XT == QTEA_E4M3) {  // (K is a multiple of 32)
    r.v = __builtin_amdgcn_raw_buffer_load_b64(xb.x, at, row_at, 0);
    r.scale = uint8_t(__builtin_amdgcn_raw_buffer_load_b8(xb.scale, in ? uint32_t(k) / 32 : kPastEnd, row_in ? uint32_t(row) * uint32_t(a.x_scale_stride) : 0u, 0));
  } else if constexpr (!ODD) {
    r.v = __builtin_amdgcn_raw_buffer_load_b128(xb.x, at, row_at, 0);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t lo = uint16_t(__builtin_amdgcn_raw_buffer_load_b16(xb.x, at + 4 * i, row_at, 0)), hi = uint16_t(__builtin_amdgcn_raw_buffer_load_b16(xb.x, at + 4 * i + 2, row_at, 0));
      r.v[i] = lo | hi << 16;
    }
  }
  return r;
}
// As 16-bit values.
template <int XT>
__device__ __forceinline__ u32x4 piece_value(const GemmArgs& a, const Piece<XT>& p, int k) {
  if constexpr (XT == QTEA_E4M3) {
    const float s = scale_of(p.scale);
    return u32x4{BF16::e4m3<false>(p.v[0], s), BF16::e4m3<true>(p.v[0], s), BF16::e4m3<false>(p.v[1], s), BF16::e4m3<true>(p.v[1], s)};
  } else {
    u32x4 v = p.v;
    if (k + 8 > a.K) {  // a row's last values: what follows them is not its own
      const int n = a.K - k;
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = 2 * i + 1 < n ? v[i] : (2 * i < n ? v[i] & 0xffffu : 0u);
    }
    return v;
  }
}

// LDS holds a unit's right operands as the lanes take them: 16-byte pieces
// [tile][CT][instruction][64 lanes], the lane within them turned by (tile, instruction)
// so that the writes, 64 consecutive pieces of a row, meet different banks.
template <int CT>
__device__ __forceinline__ uint32_t piece_at(int tile, int ct, int m, int lane) {
  return uint32_t(((tile * CT + ct) * 4 + m) * 64 + (lane ^ (m + 4 * tile)));
}
// Where the piece of `lane` in a row's 64 goes.
template <int CT>
__device__ __forceinline__ uint32_t piece_to(int row, int lane) {
  return piece_at<CT>(lane / 16, row / 16, lane & 3, (lane / 4 & 3) * 16 + (row & 15));
}

// Few strips: the waves of a workgroup share R strips' units, each with its own
// 16 rows of X, by way of LDS of its own (no barriers; a row's 64 pieces come in one
// coalesced load, where the lanes' own pieces would touch 64 lines an instruction).
// While a unit is multiplied, the next one is on its way.  Bound by start and end
// of a launch at one row (4096 x 4096 3.6 us), by bringing the activations at 16: a
// unit of them in 16 bits is 16 KB, of a strip's codes 4 (5120 x 17408, two strips
// a group: 16.4 us, 2.9 TB/s of codes and twice that of activations).  ODD: 16-bit
// loads, eight a piece, and all 16 rows whatever the batch (32000 x 5121 at 1, 16 and 40
// rows 17.5, 84 and 215 us, 32000 x 5120 16.3, 17 and 24).
template <int XT, int R, int ROWS, bool ODD>
__global__ __launch_bounds__(kThreads) void w4_gemm_split_kernel(const GemmArgs a) {
  using T = Type<XT>;
  extern __shared__ u32x4 s_x[];  // [waves][4 tiles * 4 * 64]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x >> 6)), q = lane >> 4;
  const int part = wave % a.parts;
  const int64_t group = int64_t(blockIdx.x) * (kWaves / a.parts) + wave / a.parts;
  const int64_t strip0 = min(group * R, int64_t(a.strips) - R);  // (the last groups: strips of others, again)
  const int row0 = blockIdx.y * 16;
  const XBuf xb = x_buffers<XT>(a);
  u32x4* mine = s_x + wave * (4 * 4 * 64);
  const int u0 = int(int64_t(a.units) * part / a.parts), u1 = int(int64_t(a.units) * (part + 1) / a.parts);
  f32x4 c[R];
#pragma unroll
  for (int r = 0; r < R; ++r) c[r] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  if (u0 < u1) {
    const uint8_t* codes = a.codes + strip0 * kTile;
    const uint8_t* scales = a.scales + strip0 * kUnitScales;
    u32x4 w[4][R];
    uint32_t sc[R], next[R];
    Piece<XT> x[ROWS];
    // tile j of unit u (past the last tile: that one again, times zeros)
    auto load = [&](int u, int j) {
      const uint64_t p = scalar(codes + int64_t(min(4 * u + j, a.tiles - 1)) * a.strips * kTile);
#pragma unroll
      for (int r = 0; r < R; ++r) w[j][r] = load_codes<false>(p, lane, r);
    };
    auto load_scales = [&](int u, uint32_t (&to)[R]) {
      const uint64_t p = scalar(scales + int64_t(u) * a.strips * kUnitScales);
#pragma unroll
      for (int r = 0; r < R; ++r) to[r] = load_scale4(p, lane, r);
    };
    auto load_x = [&](int u) {
#pragma unroll
      for (int i = 0; i < ROWS; ++i) x[i] = load_piece<XT, ODD>(a, xb, row0 + i, u * 512 + lane * 8);
    };
    auto write_x = [&](int u) {
      const int at = fresh(lane);
#pragma unroll
      for (int i = 0; i < ROWS; ++i) mine[piece_to<1>(i, at)] = piece_value<XT>(a, x[i], u * 512 + lane * 8);
    };
    auto multiply = [&](int j) {
      const int at = fresh(lane);
      u32x4 B[4];
#pragma unroll
      for (int m = 0; m < 4; ++m) B[m] = mine[piece_at<1>(j, 0, m, at)];
      float f[R];
#pragma unroll
      for (int r = 0; r < R; ++r) f[r] = scale_of(sc[r] >> (8 * j) & 255u);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int m = 0; m < 4; ++m)
#pragma unroll
        for (int r = 0; r < R; ++r) c[r] = T::mfma16(weights<T>(w[j][r][m], f[r]), B[m], c[r]);
    };
    load_x(u0);
    load_scales(u0, sc);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      load(u0, j);
      __builtin_amdgcn_sched_barrier(0);
    }
    write_x(u0);
    for (int u = u0; u + 1 < u1; ++u) {
      load_x(u + 1);
      load_scales(u + 1, next);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        multiply(j);
        __builtin_amdgcn_sched_barrier(0);
        load(u + 1, j);
        __builtin_amdgcn_sched_barrier(0);
      }
      write_x(u + 1);
#pragma unroll
      for (int r = 0; r < R; ++r) sc[r] = next[r];
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) multiply(j);
  }
  const int b = row0 + (lane & 15);
  if (a.parts > 1) {
    // the parts' sums, in order
    f32x4* sums = reinterpret_cast<f32x4*>(s_x);  // [waves][R][64], in the waves' own places
    f32x4* own = reinterpret_cast<f32x4*>(mine);
#pragma unroll
    for (int r = 0; r < R; ++r) own[r * 64 + lane] = c[r];
    __syncthreads();
    for (int r = part; r < R; r += a.parts) {
      const f32x4* p = sums + (wave - part) * (4 * 4 * 64) + r * 64 + lane;
      f32x4 sum = p[0];
      for (int i = 1; i < a.parts; ++i) sum += p[i * (4 * 4 * 64)];
      store_y(a, b, (strip0 + r) * 16 + 4 * q, sum);
    }
  } else {
#pragma unroll
    for (int r = 0; r < R; ++r) store_y(a, b, (strip0 + r) * 16 + 4 * q, c[r]);
  }
}

// Many strips: four a wave, its operands from LDS serve all of them.  A workgroup's waves
// share the activations there, a unit (512 columns) at a time, two units there: the
// next one is loaded while this one is multiplied, one barrier a unit.  PARTS waves
// share their strips, each has a tile or two of every unit's four, and their
// sums are added at the end: so a workgroup has four strips a wave to keep LDS
// idle enough, and as few strips altogether as give every CU its share.  HBM bounds it
// (128257 x 4096 at one row 45.5 us in a graph, 6.1 TB/s; a plain read of as many bytes
// 42), past 32 rows what a CU has to bring, decode and multiply (32000 x 5120 at 40 rows
// 24 us, 17 at 16).  STREAM: codes are loaded as used once.
template <int XT, int CT, int PARTS, bool STREAM>
__global__ __launch_bounds__(kThreads) void w4_gemm_wide_kernel(const GemmArgs a) {
  using T = Type<XT>;
  constexpr int R = kWideStrips, TILES = 4 / PARTS;  // strips of a wave, tiles of a unit
  constexpr int AHEAD = PARTS == 1 || (PARTS == 2 && CT > 2) ? 1 : 2;  // units of codes on the way, 8 or 16 KB a wave (as registers allow)
  constexpr int ROWS = CT * 16 / kWaves;             // rows of X a wave brings
  extern __shared__ u32x4 s_x[];  // [2][4 tiles * CT * 4 * 64]
  constexpr int kBuf = 4 * CT * 4 * 64;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x >> 6)), q = lane >> 4;
  const int part = wave % PARTS, tile0 = part * TILES;
  const int64_t strip0 = min((int64_t(blockIdx.x) * (kWaves / PARTS) + wave / PARTS) * R, int64_t(a.strips) - R);  // (the last waves: strips of others, again)
  const uint8_t* codes = a.codes + strip0 * kTile;
  const uint8_t* scales = a.scales + strip0 * kUnitScales;
  const XBuf xb = x_buffers<XT>(a);
  u32x4 w[AHEAD][TILES][R];
  uint32_t sc[AHEAD][R];
  auto load = [&](int s, int u, int j) {
    const uint64_t p = scalar(codes + int64_t(min(4 * u + tile0 + j, a.tiles - 1)) * a.strips * kTile);  // (past the last tile: that one again, times zeros)
#pragma unroll
    for (int r = 0; r < R; ++r) w[s][j][r] = load_codes<STREAM>(p, lane, r);
  };
  auto load_scales = [&](int s, int u) {
    const uint64_t p = scalar(scales + int64_t(min(u, a.units - 1)) * a.strips * kUnitScales);
#pragma unroll
    for (int r = 0; r < R; ++r) sc[s][r] = load_scale4(p, lane, r);
  };
  // A wave brings whole rows of a unit, 8 columns a lane.
  Piece<XT> x[AHEAD][ROWS];
  auto load_x = [&](int s, int u) {
#pragma unroll
    for (int i = 0; i < ROWS; ++i) x[s][i] = load_piece<XT, false>(a, xb, i * kWaves + wave, u * 512 + lane * 8);
  };
  auto write_x = [&](int s, int u) {
    const int at = fresh(lane);
#pragma unroll
    for (int i = 0; i < ROWS; ++i) s_x[(u & 1) * kBuf + piece_to<CT>(i * kWaves + wave, at)] = piece_value<XT>(a, x[s][i], u * 512 + lane * 8);
  };
  f32x4 c[CT][R];
#pragma unroll
  for (int t = 0; t < CT; ++t)
#pragma unroll
    for (int r = 0; r < R; ++r) c[t][r] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  // A wave's loads arrive in order, so the activations of a unit are asked for right
  // after the codes of the unit before it: whoever waits for them has those already.
  load_x(0, 0);
#pragma unroll
  for (int s = 0; s < AHEAD; ++s) {
    load_scales(s, s);
#pragma unroll
    for (int j = 0; j < TILES; ++j) load(s, s, j);
    __builtin_amdgcn_sched_barrier(0);
    if (s == 0) write_x(0, 0);
    __builtin_amdgcn_sched_barrier(0);
    load_x((s + 1) % AHEAD, s + 1);
    __builtin_amdgcn_sched_barrier(0);
  }
  __syncthreads();
  for (int u0 = 0; u0 < a.units; u0 += AHEAD) {
#pragma unroll
    for (int s = 0; s < AHEAD; ++s) {
      const int u = u0 + s;
      if (u >= a.units) break;
      const u32x4* buf = s_x + (u & 1) * kBuf;
      u32x4 B[2][CT];
      auto read_x = [&](int step) {
        const int at = fresh(lane);
#pragma unroll
        for (int t = 0; t < CT; ++t) B[step & 1][t] = buf[piece_at<CT>(tile0 + step / 4, t, step & 3, at)];
      };
      u32x4 A[2][R];
      auto decode = [&](int step) {
#pragma unroll
        for (int r = 0; r < R; ++r) A[step & 1][r] = weights<T>(w[s][step / 4][r][step & 3], scale_of(sc[s][r] >> (8 * (tile0 + step / 4)) & 255u));
      };
      read_x(0);
      decode(0);
#pragma unroll
      for (int j = 0; j < TILES; ++j) {
#pragma unroll
        for (int m = 0; m < 4; ++m) {
          const int step = 4 * j + m;
          __builtin_amdgcn_sched_barrier(0);
          if (step + 1 < 4 * TILES) read_x(step + 1), decode(step + 1);
#pragma unroll
          for (int t = 0; t < CT; ++t)
#pragma unroll
            for (int r = 0; r < R; ++r) c[t][r] = T::mfma16(A[step & 1][r], B[step & 1][t], c[t][r]);
          // the next step's operands between this one's products
          __builtin_amdgcn_sched_group_barrier(0x100, CT, 0);
#pragma unroll
          for (int i = 0; i < CT * R; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x2, (20 + CT * R - 1) / (CT * R), 0);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
        load(s, u + AHEAD, j);
        __builtin_amdgcn_sched_barrier(0);
      }
      load_scales(s, u + AHEAD);
      write_x((s + 1) % AHEAD, u + 1);  // (past the last unit: zeros)
      load_x((s + 1) % AHEAD, u + 1 + AHEAD);
      __syncthreads();
    }
  }
  if constexpr (PARTS > 1) {
    // the parts' sums, in order (LDS has room for all: 4 CT KB a wave)
    f32x4* sums = reinterpret_cast<f32x4*>(s_x);  // [waves][CT][R][64]
#pragma unroll
    for (int t = 0; t < CT; ++t)
#pragma unroll
      for (int r = 0; r < R; ++r) sums[((wave * CT + t) * R + r) * 64 + lane] = c[t][r];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < R / PARTS; ++i) {
      const int r = i * PARTS + part;
#pragma unroll
      for (int t = 0; t < CT; ++t) {
        f32x4 sum = sums[(((wave - part) * CT + t) * R + r) * 64 + lane];
#pragma unroll
        for (int k = 1; k < PARTS; ++k) sum += sums[(((wave - part + k) * CT + t) * R + r) * 64 + lane];
        store_y(a, t * 16 + (lane & 15), (strip0 + r) * 16 + 4 * q, sum);
      }
    }
  } else {
#pragma unroll
    for (int t = 0; t < CT; ++t)
#pragma unroll
      for (int r = 0; r < R; ++r) store_y(a, t * 16 + (lane & 15), (strip0 + r) * 16 + 4 * q, c[t][r]);
  }
}

}  // namespace
}  // namespace qtea_serve

using namespace qtea_serve;

namespace {

bool pack_args(const void* packed, int64_t N, int64_t K, const void* W, int type, int64_t w_stride, Layout* l, PackArgs* a) {
  if (!packed || !W || !aligned16(packed) || type < QTEA_F16 || type > QTEA_F32 || !make_layout(N, K, l)) return false;
  if (!stride_ok(w_stride, K, N) || !aligned_to_elem(W, type)) return false;
  a->w = static_cast<char*>(const_cast<void*>(W));
  a->codes = static_cast<uint8_t*>(const_cast<void*>(packed)), a->scales = a->codes + l->scales_at;
  a->stride = w_stride * elem_bytes(type), a->strips = l->strips, a->tiles = l->tiles, a->units = l->units, a->total = l->strips * l->units * 256;
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

int compute_units() {
  static std::atomic<int> known[qtea_detail::kMaxDevices];
  return qtea_detail::per_current_device(known, [](int dev) {
    int n = 0;
    return hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) == hipSuccess ? n : 0;
  });
}

using std::integral_constant;

template <int XT, int CT, int PARTS, bool STREAM>
int run_wide(const GemmArgs& a, hipStream_t st) {
  const auto kernel = w4_gemm_wide_kernel<XT, CT, PARTS, STREAM>;
  static std::atomic<int> allowed[qtea_detail::kMaxDevices];
  constexpr int lds = 2 * 4 * CT * 4 * 64 * 16, strips = kWideStrips * kWaves / PARTS;
  if (qtea_detail::allow_lds(reinterpret_cast<const void*>(kernel), lds, allowed) != hipSuccess) return QTEA_ERR_HIP;
  hipLaunchKernelGGL(kernel, dim3(uint32_t((int64_t(a.strips) + strips - 1) / strips)), dim3(kThreads), lds, st, a);
  return hipGetLastError() == hipSuccess ? QTEA_OK : QTEA_ERR_HIP;
}

template <int XT, int R, int ROWS, bool ODD>
int run_split(const GemmArgs& a, hipStream_t st) {
  const auto kernel = w4_gemm_split_kernel<XT, R, ROWS, ODD>;
  static std::atomic<int> allowed[qtea_detail::kMaxDevices];
  constexpr int lds = kWaves * 4 * 4 * 64 * 16;
  if (qtea_detail::allow_lds(reinterpret_cast<const void*>(kernel), lds, allowed) != hipSuccess) return QTEA_ERR_HIP;
  const int64_t groups = (int64_t(a.strips) + R - 1) / R;
  const int per = kWaves / a.parts;
  hipLaunchKernelGGL(kernel, dim3(uint32_t((groups + per - 1) / per), uint32_t((a.batch + 15) / 16)), dim3(kThreads), lds, st, a);
  return hipGetLastError() == hipSuccess ? QTEA_OK : QTEA_ERR_HIP;
}

// Which kernel, by strips a CU.  With five or more a wave can have whole strips
// to itself (28672 x 4096 at 16 rows of E4M3: 13.3 us, 16.0 with its columns split;
// 14336 x 4096: 11.1 and 8.8); past 16 rows with three or more, since the other
// kernel reads the weights again for each 16 (16384 x 4096 at 40 rows 18.6 us
// and 21.3).
template <int XT>
int run_gemm(GemmArgs a, int cus, hipStream_t st) {
  const int ct = (a.batch + 15) / 16;
  if (a.x_dwords && a.strips >= (ct == 1 ? 5 : 3) * cus) {
    // Strips of a workgroup: the fewest on the CU that has most, then the most.  (57344
    // x 8192 at 16 rows, 14 strips a CU: 48.7 us with workgroups of 8 strips, 44.5
    // of 16, 56.9 of 32; 28672 x 4096, 7 a CU: 13.3, 17.0, 23.4.)
    int strips = 0;
    int64_t least = INT64_MAX;
    for (const int n : {32, 16, 8}) {
      const int64_t blocks = (int64_t(a.strips) + n - 1) / n, most = (blocks + cus - 1) / cus * n;
      if (most < least && (n == 32 || blocks < (1 << 22))) least = most, strips = n;  // (a grid has 2^32 threads)
    }
    // A matrix of more than half of the Infinity Cache's 256 MB will not be there at the
    // next call, and its codes are loaded as used once: 128257 x 4096 (279 MB) at one
    // row 45.5 us for 49.9, 57344 x 8192 (250 MB) at 16 rows 43.2 for 46.3.  A smaller
    // one may be kept: 28672 x 4096 (62 MB) at one row 13.4 for 12.7 where three take
    // turns, though 13.5 for 13.9 where nine do.
    const bool stream = int64_t(a.strips) * a.tiles * kTile > (128 << 20);
    const auto with = [&](auto cols, auto past) {
      constexpr int CT = decltype(cols)::value;
      constexpr bool STREAM = decltype(past)::value;
      if (strips == 32) return run_wide<XT, CT, 1, STREAM>(a, st);
      if (strips == 16) return run_wide<XT, CT, 2, STREAM>(a, st);
      return run_wide<XT, CT, 4, STREAM>(a, st);
    };
    const auto by_cols = [&](auto past) {
      if (ct == 1) return with(integral_constant<int, 1>(), past);
      if (ct == 2) return with(integral_constant<int, 2>(), past);
      return ct == 3 ? with(integral_constant<int, 3>(), past) : with(integral_constant<int, 4>(), past);
    };
    return stream ? by_cols(std::true_type()) : by_cols(std::false_type());
  }
  // Strips a group: the most that leave groups for six CUs of ten (10240 x 8192 at 16
  // rows 12.5 us with four, 16.2 with two; 8192 x 28672: 37.5 with four, that is
  // half of the CUs, 30.5 with two); waves a group: eight a CU, if there are units.
  int R = a.x_dwords ? 4 : 2;
  while (R > 1 && (a.strips < R || int64_t(a.strips) * ct * 10 < int64_t(R) * 6 * cus)) R /= 2;
  a.parts = 1;
  while (a.parts < kWaves && a.parts < a.units && (int64_t(a.strips) + R - 1) / R * a.parts < 8 * int64_t(cus)) a.parts *= 2;
  const auto with = [&](auto strips) {
    constexpr int RR = decltype(strips)::value;
    if constexpr (XT != QTEA_E4M3 && RR < 4) {
      if (!a.x_dwords) return run_split<XT, RR, 16, true>(a, st);
    }
    if (a.batch == 1) return run_split<XT, RR, 1, false>(a, st);
    if (a.batch <= 4) return run_split<XT, RR, 4, false>(a, st);
    if (a.batch <= 8) return run_split<XT, RR, 8, false>(a, st);
    return run_split<XT, RR, 16, false>(a, st);
  };
  if (R == 4) return with(integral_constant<int, 4>());
  return R == 2 ? with(integral_constant<int, 2>()) : with(integral_constant<int, 1>());
}

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
  if (y_type < QTEA_F16 || y_type > QTEA_F32 || !aligned_to_elem(Y, y_type) || !stride_ok(y_stride, N, batch) || !stride_ok(x_stride, K, batch)) return QTEA_ERR_INVALID_ARG;
  if (x_type == QTEA_E4M3) {
    if (K % 32 != 0 || !rows_aligned16(X, x_stride, x_type) || !x_scale || !stride_ok(x_scale_stride, K / 32, batch)) return QTEA_ERR_INVALID_ARG;
  } else if ((x_type != QTEA_F16 && x_type != QTEA_BF16) || x_scale || !aligned_to_elem(X, x_type)) {
    return QTEA_ERR_INVALID_ARG;
  }
  if (packed_bytes < l.bytes) return QTEA_ERR_WORKSPACE;
  GemmArgs a;
  a.codes = static_cast<const uint8_t*>(packed), a.scales = a.codes + l.scales_at;
  a.x = static_cast<const char*>(X), a.x_scale = x_scale, a.y = static_cast<char*>(Y);
  a.x_stride = x_stride * elem_bytes(x_type), a.x_scale_stride = x_scale_stride, a.y_stride = y_stride * elem_bytes(y_type);
  a.N = int32_t(N), a.K = int32_t(K), a.strips = int32_t(l.strips), a.tiles = int32_t(l.tiles), a.units = int32_t(l.units);
  a.batch = batch, a.y_type = y_type;
  const int64_t x_bytes = (batch - 1) * a.x_stride + K * elem_bytes(x_type), sc_bytes = x_scale ? (batch - 1) * x_scale_stride + K / 32 : 0;
  if (x_bytes > (1 << 30) || sc_bytes > (1 << 30)) return QTEA_ERR_INVALID_ARG;
  // (a last dword may be half X's: the other half is read and not used)
  a.x_bytes = int32_t((x_bytes + 3) & ~int64_t(3)), a.x_scale_bytes = int32_t(sc_bytes);
  a.x_dwords = x_type == QTEA_E4M3 || ((reinterpret_cast<uintptr_t>(X) | (batch > 1 ? uint64_t(a.x_stride) : 0)) % 4 == 0);
  if (!a.x_dwords) a.x_bytes = int32_t(x_bytes);
  a.y_wide = (reinterpret_cast<uintptr_t>(Y) | uint64_t(a.y_stride)) % 8 == 0;
  const int cus = compute_units();
  if (cus == 0) return QTEA_ERR_HIP;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  if (x_type == QTEA_F16) return run_gemm<QTEA_F16>(a, cus, st);
  if (x_type == QTEA_BF16) return run_gemm<QTEA_BF16>(a, cus, st);
  return run_gemm<QTEA_E4M3>(a, cus, st);
}

}  // extern "C"
