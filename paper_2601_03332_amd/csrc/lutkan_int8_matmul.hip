// Products of 8-bit integer codes with a scale for each row of both operands:
//   y[s][n] = x_scale[s] * w_scale[n] * sum_k x[s][k] * w[n][k]
// for one weight, or for rows grouped by expert with a weight each.  The sums are whole numbers and stay in the matrix instructions' 32-bit
// accumulators from the first k to the last (k < 2^17: no sum of products of (-128)^2 overflows), so that their order does not matter.
//
// The weight is the instruction's first operand and the activations its second: a lane holds runs of four neighbouring outputs of one row.  Both
// operands are read in the same order along k, so which k an instruction takes first does not matter.
#include "lutkan_product.h"

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

__device__ __forceinline__ i32x4 product_16x16(u32x4 w, u32x4 x, i32x4 sum) {            // 64 of k
  return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, w), __builtin_bit_cast(i32x4, x), sum, 0, 0, 0);
}
__device__ __forceinline__ i32x16 product_32x32(u32x4 w, u32x4 x, i32x16 sum) {          // 32 of k
  return __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(i32x4, w), __builtin_bit_cast(i32x4, x), sum, 0, 0, 0);
}

// Scales that fp32 multiplies without loss: a sum below 2^31 times two of them lies beyond fp32 only where y does.
__device__ __forceinline__ bool ordinary(float scale) { return scale >= 0x1p-60f && scale <= 0x1p60f; }

// Four sums times the row's scale, then times their own, each rounded; in fp64 where one of the two scales is not ordinary (`any`: some are).  Every kernel does
// it so, and the sums are exact: an output does not depend on the kernel.
__device__ __forceinline__ f32x4 scaled(i32x4 sum, float x_scale, f32x4 w_scale, bool any) {
  f32x4 v;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    v[e] = (float)sum[e] * x_scale * w_scale[e];
    if (any && !(ordinary(x_scale) && ordinary(w_scale[e]))) v[e] = (float)((double)sum[e] * ((double)x_scale * (double)w_scale[e]));
  }
  return v;
}

// The scales of four neighbouring outputs, those that exist; 1 for others.
__device__ __forceinline__ f32x4 weight_scales(const ProductArgs &a, int group, int col) {
  const float *p = a.w_scales + (int64_t)group * a.n + col;
  if (col + 4 <= a.n) return load_any<f32x4>(p);
  f32x4 v{1.0f, 1.0f, 1.0f, 1.0f};
#pragma unroll
  for (int e = 0; e < 4; ++e) if (col + e < a.n) v[e] = p[e];
  return v;
}

// A work-group computes 16 MT rows x 16 NT columns from global memory straight into registers; its waves take the blocks of k in turn,
// and their sums meet in LDS.
// Bound by what it reads, as no work-group shares with another: 16 rows of 4096 -> 4096 7.1 us replayed with 16 x 16 (256 work-groups, one to a compute unit;
// weights 17 MB and as much of x again), 8.9 with 16 x 32; one row 5.8.
template <int MT, int NT, bool GROUPED, bool ALIGNED>
__global__ __launch_bounds__(1024) void lutkan_int8_direct_kernel(const ProductArgs a) {
  extern __shared__ __align__(16) i32x4 s_part[];                // [wave][row tile][column tile][lane]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = a.extent;
  const int p = lane >> 4, col0 = blockIdx.x * (16 * NT);
  RowTile t;
  if constexpr (GROUPED) {
    t = grouped_tile<16 * MT>(a, [&](int tiles) { return (int)blockIdx.y < tiles ? (int)blockIdx.y : -1; });
    if (t.end <= t.first) return;
  } else {
    t.first = (int64_t)blockIdx.y * (16 * MT);
    t.end = min(t.first + 16 * MT, (int64_t)a.rows);
    t.group = 0;
  }
  i32x4 acc[MT][NT];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[m][n] = i32x4{0, 0, 0, 0};
  int64_t from[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) from[m] = t.group < 0 ? -1 : source_row<GROUPED>(a, min(t.first + 16 * m + (lane & 15), t.end - 1));
  float xs[MT];                                                  // (asked for before the codes: at the end they would be waited for)
  f32x4 ws[NT];
#pragma unroll
  for (int m = 0; m < MT; ++m) xs[m] = from[m] >= 0 ? a.x_scales[from[m] * a.x_scales_stride] : 1.0f;
#pragma unroll
  for (int n = 0; n < NT; ++n) ws[n] = weight_scales(a, max(t.group, 0), col0 + 16 * n + 4 * p);
  if (t.group >= 0) {
    const unsigned char *x[MT], *w[NT];
#pragma unroll
    for (int m = 0; m < MT; ++m) x[m] = a.x + max(from[m], (int64_t)0) * a.x_stride;
#pragma unroll
    for (int n = 0; n < NT; ++n) w[n] = a.w + t.group * a.w_matrix_stride + (int64_t)min(col0 + 16 * n + (lane & 15), a.n - 1) * a.w_stride;
    // kDepth blocks are read before the first is multiplied.
    constexpr int kDepth = MT * NT == 1 ? 4 : MT * NT == 2 ? 2 : 1;
    struct Block { Piece<ALIGNED> w[NT][2], x[MT][2]; };
    const auto read = [&](Block &to, int b) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int n = 0; n < NT; ++n) to.w[n][h].read(w[n] + b * kScaleBlock + 64 * h + 16 * p);
#pragma unroll
        for (int m = 0; m < MT; ++m) to.x[m][h].read(x[m] + b * kScaleBlock + 64 * h + 16 * p);
      }
    };
    const auto multiply = [&](const Block &of) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int n = 0; n < NT; ++n) acc[m][n] = product_16x16(of.w[n][h].get(low_bits(w[n])), of.x[m][h].get(low_bits(x[m])), acc[m][n]);
    };
    const int whole = a.k / kScaleBlock;
    // The work-groups of an XCD begin at different blocks, so that they do not all ask for the same lines of x at a time.
    const int shift = whole ? (int)(blockIdx.x / 8 % (unsigned)whole) : 0;
    const auto turn = [&](int b) { return b + shift < whole ? b + shift : b + shift - whole; };
    for (int b = wave; b < whole; b += waves * kDepth) {
      Block held[kDepth];
#pragma unroll
      for (int d = 0; d < kDepth; ++d) if (b + d * waves < whole) read(held[d], turn(b + d * waves));
#pragma unroll
      for (int d = 0; d < kDepth; ++d) if (b + d * waves < whole) multiply(held[d]);
    }
    if (whole < a.k_blocks() && whole % waves == wave) {         // the last block, not whole
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int k0 = whole * kScaleBlock + 64 * h + 16 * p;
        u32x4 wc[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) wc[n] = piece_at_end(w[n], k0, a.k);
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          const u32x4 xc = piece_at_end(x[m], k0, a.k);
#pragma unroll
          for (int n = 0; n < NT; ++n) acc[m][n] = product_16x16(wc[n], xc, acc[m][n]);
        }
      }
    }
  }
  if (waves > 1) {
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int n = 0; n < NT; ++n) s_part[((wave * MT + m) * NT + n) * 64 + lane] = acc[m][n];
    __syncthreads();
  }
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      if ((m * NT + n) % waves != wave) continue;                // a wave sums every waves-th tile
      i32x4 v = acc[m][n];
      if (waves > 1) {
        v = s_part[(m * NT + n) * 64 + lane];
        for (int o = 1; o < waves; ++o) v += s_part[((o * MT + m) * NT + n) * 64 + lane];
      }
      const int64_t row = t.first + 16 * m + (lane & 15);
      const int col = col0 + 16 * n + 4 * p;
      f32x4 y{0.0f, 0.0f, 0.0f, 0.0f};
      const bool any = !__all(ordinary(xs[m]) && ordinary(ws[n][0]) && ordinary(ws[n][1]) && ordinary(ws[n][2]) && ordinary(ws[n][3]));
      if (from[m] >= 0) y = scaled(v, xs[m], ws[n], any);
      if (row < t.end) store_outputs(a, row, col, y);
    }
}

template <int MT, int NT, bool GROUPED>
int launch_direct(ProductArgs a, int64_t row_tiles, bool aligned, const char *who, hipStream_t s) {
  if (row_tiles > 65535) return fail(LUTKAN_EUNSUPPORTED, "%s: too many rows", who);
  const int waves = a.extent = std::min(a.k_blocks(), 16);
  const dim3 grid((unsigned)((a.n + 16 * NT - 1) / (16 * NT)), (unsigned)row_tiles);
  lutkan::plan_note("int8_direct rows=%d columns=%d waves=%d; ", 16 * MT, 16 * NT, waves);
  const auto kernel = aligned ? lutkan_int8_direct_kernel<MT, NT, GROUPED, true> : lutkan_int8_direct_kernel<MT, NT, GROUPED, false>;
  hipLaunchKernelGGL(kernel, grid, dim3(64 * waves), waves > 1 ? (size_t)waves * MT * NT * 64 * sizeof(i32x4) : 0, s, a);
  return check_launch(who);
}

// The outputs of a wave's 32 TM rows x 32 TN columns.  A lane's sixteen sums of 32 x 32 are columns 8 g + 4 h + e of row lane % 32 (g < 4, h = lane / 32, e < 4):
// 32 rows at a time change places through LDS, so that neighbouring lanes hold neighbouring outputs, 16 bytes each, and a store covers whole
// rows of the tile.  (Stored from where they lie, the code is as long as the sums are many: 13000 lines for the largest tile, which took longer to fetch than
// its stores to run.  8192 rows of 64 -> 4096 into bf16 49 us; 27 so; 21 with the tile that it gets now.)
constexpr int dump_pitch(int TN) { return 32 * TN * 4 + 16; }    // bytes of a row there
constexpr int dump_bytes(int TN) { return 32 * dump_pitch(TN); }

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
template <int TYPE>
__device__ __forceinline__ unsigned two_outputs(float a, float b) {
  if constexpr (TYPE == LUTKAN_BF16) return __builtin_bit_cast(unsigned, bf16x2{(__bf16)a, (__bf16)b});
  else return f16_bits(a) | (f16_bits(b) << 16);
}

// Four (32 bits) or eight (16 bits) neighbouring outputs of a row.
template <int TYPE, int N>
__device__ __forceinline__ void store_some(const ProductArgs &a, int64_t row, int col, const f32x4 (&v)[N]) {
  if constexpr (TYPE == LUTKAN_F32) {
    store_outputs(a, row, col, v[0]);
  } else {
    unsigned char *to = a.y + (row * a.y_stride + col) * 2;
    const u32x4 eight{two_outputs<TYPE>(v[0][0], v[0][1]), two_outputs<TYPE>(v[0][2], v[0][3]), two_outputs<TYPE>(v[1][0], v[1][1]), two_outputs<TYPE>(v[1][2], v[1][3])};
    if (col + 8 <= a.n) { store_any(to, eight); return; }
#pragma unroll
    for (int e = 0; e < 8; ++e) if (col + e < a.n) store_any(to + 2 * e, (unsigned short)(eight[e >> 1] >> ((e & 1) * 16)));
  }
}

// What they are scaled with, asked for before the codes: at the end it would be waited for.
template <int TM, int TN, bool GROUPED>
struct WaveScales {
  float xs[TM];                                                  // of row 32 m + lane % 32; 0: a row of zeros
  f32x4 ws[2];                                                   // of the lane's columns (store_wave)
  bool fine = true;
  __device__ __forceinline__ WaveScales(const ProductArgs &a, const RowTile &t, int64_t row0, int col0) {
    const int lane = threadIdx.x & 63, cols = a.y_type == LUTKAN_F32 ? 4 : 8, col = col0 + lane * cols % (32 * TN);
#pragma unroll
    for (int m = 0; m < TM; ++m) {
      const int64_t from = t.group < 0 ? -1 : source_row<GROUPED>(a, min(row0 + 32 * m + (lane & 31), t.end - 1));
      xs[m] = from >= 0 ? a.x_scales[from * a.x_scales_stride] : 0.0f;
      fine = fine && (from < 0 || ordinary(xs[m]));
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) ws[i] = weight_scales(a, max(t.group, 0), col + 4 * i);
  }
};

template <int TYPE, int TM, int TN, bool GROUPED>
__device__ __forceinline__ void store_wave(const ProductArgs &a, const RowTile &t, const i32x16 (&acc)[TM][TN], int64_t row0, int col0, unsigned char *dump, const WaveScales<TM, TN, GROUPED> &scales) {
  constexpr int kCols = TYPE == LUTKAN_F32 ? 4 : 8, kLanes = 32 * TN / kCols, kRows = 64 / kLanes;       // columns of a lane, lanes of a row, rows at a time
  const int lane = threadIdx.x & 63, col = col0 + lane % kLanes * kCols;
  const int64_t last = t.end - 1;
  const auto &xs = scales.xs;
  const auto &ws = scales.ws;
  bool fine = scales.fine;
#pragma unroll
  for (int i = 0; i < kCols / 4; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) fine = fine && ordinary(ws[i][e]);
  const bool exact = !__all(fine);                               // (then the sums change places, and not their products with xs)
  unsigned char *const to = dump + (lane & 31) * dump_pitch(TN) + (lane >> 5) * 16;
  const unsigned char *const from = dump + lane / kLanes * dump_pitch(TN) + lane % kLanes * kCols * 4;
#pragma unroll
  for (int m = 0; m < TM; ++m) {
    const bool none = xs[m] == 0.0f;
#pragma unroll
    for (int n = 0; n < TN; ++n)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        i32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float product = none ? 0.0f : (float)acc[m][n][4 * g + e] * xs[m];
          v[e] = exact ? acc[m][n][4 * g + e] : (int)__float_as_uint(product);
        }
        *reinterpret_cast<i32x4 *>(to + (32 * n + 8 * g) * 4) = v;
      }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (!exact) {
      constexpr int kParts = 32 / kRows < 4 ? 32 / kRows : 4;
#pragma unroll 1
      for (int r0 = 0; r0 < 32; r0 += kParts * kRows) {
        f32x4 v[kParts][kCols / 4];
#pragma unroll
        for (int o = 0; o < kParts; ++o)
#pragma unroll
          for (int i = 0; i < kCols / 4; ++i) v[o][i] = *reinterpret_cast<const f32x4 *>(from + (r0 + o * kRows) * dump_pitch(TN) + 16 * i);
#pragma unroll
        for (int o = 0; o < kParts; ++o) {
#pragma unroll
          for (int i = 0; i < kCols / 4; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) v[o][i][e] *= ws[i][e];
          const int64_t row = row0 + 32 * m + r0 + o * kRows + lane / kLanes;
          if (row <= last && col < a.n) store_some<TYPE>(a, row, col, v[o]);
        }
      }
    } else {
#pragma unroll 1
      for (int r0 = 0; r0 < 32; r0 += kRows) {
        const int64_t row = row0 + 32 * m + r0 + lane / kLanes, source = t.group < 0 ? -1 : source_row<GROUPED>(a, min(row, last));
        const float x_scale = source < 0 ? 0.0f : a.x_scales[source * a.x_scales_stride];
        f32x4 v[kCols / 4];
#pragma unroll
        for (int i = 0; i < kCols / 4; ++i) {
          v[i] = scaled(*reinterpret_cast<const i32x4 *>(from + r0 * dump_pitch(TN) + 16 * i), x_scale, ws[i], true);
          if (source < 0) v[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }
        if (row <= last && col < a.n) store_some<TYPE>(a, row, col, v);
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");      // the next rows come behind the reads of these
  }
}

template <int N>
__device__ __forceinline__ void wait_vector_loads() { __builtin_amdgcn_s_waitcnt(0x0f70 | (N & 15) | (N >> 4 << 14)); }      // vmcnt(N)

// A tile of 32 TM WM rows x 32 TN WN columns for a work-group of KG teams of WM x WN waves, each wave 32 TM rows x 32 TN columns of it.  The teams
// take the blocks of k in turn; their sums meet in LDS.  A team's blocks go through LDS, in several buffers.  A row's 16-byte pieces lie in an
// order that depends on the row (piece_at), so that the 16 rows that a read of 16 lanes takes lie in different banks.
//   A block is multiplied in steps of 32 k.  While one is, the next one's fragments are read, and copies of a later block go out; only the last
//   step has to know that all waves have read the block and that the next one is there, and its fragments have been read before.
//   ASYNC: the pieces go from global memory to LDS without passing through registers: needs rows at dword addresses and offsets that fit 32 bits.  Blocks
//   of 64 k in five buffers: four are on their way while one is multiplied.
//   Otherwise, and for a last block that is not whole, through registers: blocks of 128 k in two buffers.
// What it measured, into bf16, three sets of inputs in turn: 8192 rows of 4096 -> 4096 with 256 x 256 125 - 133 us (2.1 - 2.2 POP/s; a library product of such codes,
// into int32, 131), 128 x 256 148, 128 x 128 171.  Matrix cores 0.55 busy at 1.8 GHz: power decides (codes of zeros 97 us; without the copies 138 where it
// took 152, without the fragments' reads 150), then the ends of the two rounds, 21 us.  128 x 128 and smaller wait for the copies, 16 TB/s over the GPU.
template <int TM, int TN, int WM, int WN, int KG, bool ASYNC>
struct Tile {
  static constexpr int kRows = 32 * TM * WM, kCols = 32 * TN * WN, kThreads = 64 * WM * WN;
  static constexpr int kBlock = ASYNC ? 64 : 128, kStage = (kRows + kCols) * kBlock, kHalf = lutkan::kLdsPerWorkGroup / 2;
  static constexpr int kStages = !ASYNC ? 2 : KG * 5 * kStage <= kHalf || WM * WN * KG > 4 ? 5 : kHalf / kStage;
  static constexpr int kParts = KG > 1 ? (KG - 1) * kRows * kCols * 4 : 0;       // the sums of all teams but the one that adds them up
  static constexpr int kLds = std::max(KG * kStages * kStage, kParts + WM * WN * dump_bytes(TN));
  static_assert(kLds <= lutkan::kLdsPerWorkGroup, "LDS");
};

template <int TM, int TN, int WM, int WN, int KG, bool GROUPED, bool ASYNC>
__global__ __launch_bounds__(64 * WM * WN * KG, WM * WN * KG >= 16 ? 4 : 2) void lutkan_int8_tiled_kernel(const ProductArgs a) {
  using T = Tile<TM, TN, WM, WN, KG, ASYNC>;
  constexpr int kRows = T::kRows, kCols = T::kCols, kWaves = WM * WN, kBlock = T::kBlock, kStages = T::kStages, kStage = T::kStage, kSteps = kBlock / 32, kPieces = kBlock / 16;
  constexpr int kCopyRows = 1024 / kBlock, kXCopies = kRows / kCopyRows / kWaves, kWCopies = kCols / kCopyRows / kWaves, kCopies = kXCopies + kWCopies;     // for each wave
  static_assert(kXCopies * kCopyRows * kWaves == kRows && kWCopies * kCopyRows * kWaves == kCols && 16 % kCopyRows == 0 && kXCopies * kCopyRows % 16 == 0 && kWCopies * kCopyRows % 16 == 0, "copies");
  extern __shared__ __align__(16) unsigned char s_tiles[];       // [team][buffer][rows of x, rows of the weight][kBlock]
  const int lane = threadIdx.x & 63, wave_of_all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), team = wave_of_all / kWaves;
  const int wave = wave_of_all % kWaves, wm = wave / WN, wn = wave % WN, h = lane >> 5;
  // Work-groups go to the eight XCDs in turn: each XCD gets a run of neighbouring tiles, and in a run eight row tiles share a column
  // tile before the next, so that what an XCD's work-groups read at a time meets in its L2.
  const unsigned col_tiles = (a.n + kCols - 1) / kCols;
  int col0 = 0;
  const auto tile_of = [&](unsigned row_tiles) {                 // the row tile; sets the column
    const unsigned tiles = row_tiles * col_tiles;
    if (blockIdx.x >= tiles) return -1;
    const unsigned xcd = blockIdx.x % 8, of_xcd = tiles / 8, more = tiles % 8;
    const unsigned tile = xcd * of_xcd + min(xcd, more) + blockIdx.x / 8;
    const unsigned band = tile / (8 * col_tiles), in_band = tile - band * 8 * col_tiles, high = min(8u, row_tiles - band * 8);
    col0 = (int)(in_band / high) * kCols;
    return (int)(band * 8 + in_band % high);
  };
  RowTile t;
  if constexpr (GROUPED) {
    t = grouped_tile<kRows>(a, tile_of);
  } else {
    t.first = (int64_t)tile_of(a.extent) * kRows;               // (the grid has as many work-groups as there are tiles)
    t.end = min(t.first + kRows, (int64_t)a.rows);
    t.group = 0;
  }
  if (t.end <= t.first) return;
  const int64_t row0 = t.first + wm * TM * 32;
  const int wave_col0 = col0 + wn * TN * 32;
  const WaveScales<TM, TN, GROUPED> scales(a, t, row0, wave_col0);
  i32x16 acc[TM][TN];
#pragma unroll
  for (int m = 0; m < TM; ++m)
#pragma unroll
    for (int n = 0; n < TN; ++n) acc[m][n] = i32x16{0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
  if (t.group >= 0) {
    const auto uniform = [](const unsigned char *p) {            // (the copies take it from scalar registers)
      const uint64_t at = reinterpret_cast<uint64_t>(p);
      const unsigned high = __builtin_amdgcn_readfirstlane((unsigned)(at >> 32)), low = __builtin_amdgcn_readfirstlane((unsigned)at);     // (unsigned: the builtin's result is signed)
      return reinterpret_cast<const unsigned char *>((uint64_t)high << 32 | low);
    };
    const unsigned char *w_tile = uniform(a.w + t.group * a.w_matrix_stride + (int64_t)col0 * a.w_stride);
    const unsigned char *x_tile = uniform(GROUPED ? a.x : a.x + t.first * a.x_stride);
    // Piece `piece` of row `row` lies at this place of the row's kPieces (its own inverse).
    const auto piece_at = [](int row, int piece) { return piece ^ (row / (16 / kPieces) & (kPieces - 1)); };
    const int copy_row = lane / kPieces;                         // a lane's row of a copy, and the columns of its piece: the same for every 16 rows
    const auto copy_from = [&](int c) { return piece_at(c * kCopyRows + copy_row, lane % kPieces) * 16; };
    typedef std::conditional_t<ASYNC, unsigned, int64_t> offset_t;
    offset_t x_from[kXCopies], w_from[kWCopies];                 // the rows that this lane's pieces come from
    const auto row_of = [&](int r) {                             // rows behind the last are the last again
      const int64_t row = min(t.first + r, t.end - 1);
      return GROUPED ? max(source_row<GROUPED>(a, row), (int64_t)0) : row - t.first;
    };
#pragma unroll
    for (int c = 0; c < kXCopies; ++c) x_from[c] = (offset_t)(row_of((wave * kXCopies + c) * kCopyRows + copy_row) * a.x_stride) + (ASYNC ? copy_from(c) : 0);
#pragma unroll
    for (int c = 0; c < kWCopies; ++c) w_from[c] = (offset_t)((int64_t)min((wave * kWCopies + c) * kCopyRows + copy_row, a.n - 1 - col0) * a.w_stride) + (ASYNC ? copy_from(c) : 0);
    const int whole = a.k / kBlock, own = (whole - team + KG - 1) / KG, blocks = (whole + KG - 1) / KG;     // whole blocks: all, this team's, the first team's
    unsigned char *const s_team = s_tiles + team * (kStages * kStage);
    const auto stage = [&](int block) { return s_team + block % kStages * kStage; };
    Piece<false> held[ASYNC ? 1 : kCopies];                      // (without ASYNC: rows at any address)
    // Copy c of this team's block: on its way into its buffer, or asked for until put() puts it there.
    const auto ask = [&](int block, unsigned char *to, int c) {
      const bool of_x = c < kXCopies;
      const int cw = c - kXCopies;
      const int64_t k0 = (int64_t)(block * KG + team) * kBlock;
      if constexpr (ASYNC) copy16_global_to_lds_at((of_x ? x_tile : w_tile) + k0, of_x ? x_from[c] : w_from[cw], to + (of_x ? (wave * kXCopies + c) * 1024 : kRows * kBlock + (wave * kWCopies + cw) * 1024));
      else held[c].read((of_x ? x_tile + x_from[c] : w_tile + w_from[cw]) + (k0 + copy_from(of_x ? c : cw)));
    };
    const auto put = [&](int block) {
      if constexpr (!ASYNC) {
        unsigned char *to = stage(block) + lane * 16;
#pragma unroll
        for (int c = 0; c < kXCopies; ++c) *reinterpret_cast<u32x4 *>(to + (wave * kXCopies + c) * 1024) = held[c].get(low_bits(x_tile + x_from[c]));
#pragma unroll
        for (int c = 0; c < kWCopies; ++c) *reinterpret_cast<u32x4 *>(to + kRows * kBlock + (wave * kWCopies + c) * 1024) = held[kXCopies + c].get(low_bits(w_tile + w_from[c]));
      }
    };
    // The last block, if it is not whole: this team's block `own`.
    const auto put_end = [&]() {
      unsigned char *to = stage(own) + lane * 16;
      for (int c = 0; c < kXCopies; ++c)
        *reinterpret_cast<u32x4 *>(to + (wave * kXCopies + c) * 1024) = piece_at_end(x_tile + (x_from[c] - (ASYNC ? copy_from(c) : 0)), whole * kBlock + copy_from(c), a.k);
      for (int c = 0; c < kWCopies; ++c)
        *reinterpret_cast<u32x4 *>(to + kRows * kBlock + (wave * kWCopies + c) * 1024) = piece_at_end(w_tile + (w_from[c] - (ASYNC ? copy_from(c) : 0)), whole * kBlock + copy_from(c), a.k);
    };
    int at_piece[kSteps];                                        // a lane's bytes of a 32-row subtile, by step of 32 k
#pragma unroll
    for (int q = 0; q < kSteps; ++q) at_piece[q] = (lane & 31) * kBlock + piece_at(lane & 31, 2 * q + h) * 16;
    u32x4 xf[2][TM], wf[2][TN];
    // Fragment f of step q of a block, into buffer q & 1.
    const auto read = [&](const unsigned char *of, int q, int f) {
      const unsigned char *from = of + at_piece[q] + (f < TM ? (wm * TM + f) * 32 * kBlock : (kRows + (wn * TN + f - TM) * 32) * kBlock);
      if (f < TM) xf[q & 1][f] = *reinterpret_cast<const u32x4 *>(from);
      else wf[q & 1][f - TM] = *reinterpret_cast<const u32x4 *>(from);
    };
    constexpr int kFirst = kCopies / 2, kLast = kSteps - 1;      // of a block's copies go out behind the barrier, the others a step later
    // Step q: its products, and between them READS fragments of the next step and ASKS copies of a block, from copy `first_ask` on.
    const auto multiply = [&](auto q_, auto reads_, auto asks_, const unsigned char *read_from, int ask_block, int first_ask) {
      constexpr int q = decltype(q_)::value, kReads = decltype(reads_)::value, kOps = kReads + decltype(asks_)::value, kAll = TM * TN;
      unsigned char *const to = kOps > kReads ? stage(ask_block) : nullptr;
#pragma unroll
      for (int i = 0; i < kAll; ++i) {
#pragma unroll
        for (int o = i * kOps / kAll; o < (i + 1) * kOps / kAll; ++o) {
          if (o < kReads) read(read_from, (q + 1) % kSteps, o);
          else ask(ask_block, to, first_ask + o - kReads);
        }
        __builtin_amdgcn_sched_barrier(0);
        acc[i / TN][i % TN] = product_32x32(wf[q & 1][i % TN], xf[q & 1][i / TN], acc[i / TN][i % TN]);
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    // A block with `after` more behind it, at most kStages of which matter: of those, the next one has to be there at its last step, the copies of the
    // last one in flight go out in two parts.
    const auto multiply_block = [&](int block, auto after_) {
      constexpr int kAfter = decltype(after_)::value, kAhead = kStages - 1;
      constexpr std::integral_constant<int, TM + TN> reads{};
      constexpr std::integral_constant<int, 0> none{};
      multiply(std::integral_constant<int, 0>(), reads, std::integral_constant<int, (kAfter >= kAhead ? kCopies - kFirst : 0)>(), stage(block), block + kAhead, kFirst);
      if constexpr (kSteps == 4) {
        multiply(std::integral_constant<int, 1>(), reads, none, stage(block), 0, 0);
        multiply(std::integral_constant<int, 2>(), reads, none, stage(block), 0, 0);
      }
      wait_vector_loads<(ASYNC && kAfter > 1 ? std::min(kAfter, kAhead) - 1 : 0) * kCopies>();
      if constexpr (kAfter > 0) put(block + 1);
      lds_barrier();                                             // the next block is there, and nobody reads this one any more
      multiply(std::integral_constant<int, kLast>(), std::integral_constant<int, (kAfter > 0 ? TM + TN : 0)>(), std::integral_constant<int, (kAfter > kAhead ? kFirst : 0)>(), stage(block + 1),
               block + kStages, 0);
    };
    if constexpr (ASYNC) {
#pragma unroll
      for (int b = 0; b < kStages - 1; ++b)
        if (b < own)
#pragma unroll
          for (int c = 0; c < kCopies; ++c) ask(b, stage(b), c);
      if (kStages - 1 < own) {
#pragma unroll
        for (int c = 0; c < kFirst; ++c) ask(kStages - 1, stage(kStages - 1), c);
        wait_vector_loads<(kStages - 2) * kCopies + kFirst>();
      } else {
        wait_all_vector_loads();
      }
    } else {
      if (own > 0) {
#pragma unroll
        for (int c = 0; c < kCopies; ++c) ask(0, nullptr, c);
        put(0);
      }
      if (own > 1) {
#pragma unroll
        for (int c = 0; c < kFirst; ++c) ask(1, nullptr, c);
      }
    }
    lds_barrier();
    if (own > 0) {
#pragma unroll
      for (int f = 0; f < TM + TN; ++f) read(stage(0), 0, f);
    }
    int block = 0;
    for (; block + kStages < own; ++block) multiply_block(block, std::integral_constant<int, kStages>());
    if constexpr (kStages > 4) {
      if (block + 4 < own) multiply_block(block++, std::integral_constant<int, 4>());
    }
    if constexpr (kStages > 3) {
      if (block + 3 < own) multiply_block(block++, std::integral_constant<int, 3>());
    }
    if constexpr (kStages > 2) {
      if (block + 2 < own) multiply_block(block++, std::integral_constant<int, 2>());
    }
    if (block + 1 < own) multiply_block(block++, std::integral_constant<int, 1>());
    if (block < own) multiply_block(block++, std::integral_constant<int, 0>());
    for (; block < blocks; ++block) lds_barrier();               // (a team with a block less than the first)
    if (whole * kBlock < a.k) {
      const bool mine = whole % KG == team;
      if (mine) put_end();                                       // (into a buffer that nobody reads since the last barrier)
      lds_barrier();
      if (mine) {
#pragma unroll
        for (int q = 0; q < kSteps; ++q) {
#pragma unroll
          for (int f = 0; f < TM + TN; ++f) read(stage(own), q, f);
#pragma unroll
          for (int i = 0; i < TM * TN; ++i) acc[i / TN][i % TN] = product_32x32(wf[q & 1][i % TN], xf[q & 1][i / TN], acc[i / TN][i % TN]);
        }
      }
    }
    if constexpr (KG > 1) {
      lds_barrier();                                             // nobody reads the buffers any more
      i32x4 *parts = reinterpret_cast<i32x4 *>(s_tiles);         // [team - 1][wave][m][n][quarter][lane]
      const auto place = [&](int of, int m, int n, int g) { return ((((of * kWaves + wave) * TM + m) * TN + n) * 4 + g) * 64 + lane; };
      if (team > 0) {
#pragma unroll
        for (int m = 0; m < TM; ++m)
#pragma unroll
          for (int n = 0; n < TN; ++n)
#pragma unroll
            for (int g = 0; g < 4; ++g) parts[place(team - 1, m, n, g)] = i32x4{acc[m][n][4 * g], acc[m][n][4 * g + 1], acc[m][n][4 * g + 2], acc[m][n][4 * g + 3]};
      }
      lds_barrier();
      if (team > 0) return;
#pragma unroll
      for (int m = 0; m < TM; ++m)
#pragma unroll
        for (int n = 0; n < TN; ++n)
#pragma unroll
          for (int g = 0; g < 4; ++g)
            for (int o = 0; o < KG - 1; ++o) {
              const i32x4 part = parts[place(o, m, n, g)];
#pragma unroll
              for (int e = 0; e < 4; ++e) acc[m][n][4 * g + e] += part[e];
            }
    }
  }
  if (KG > 1 && team > 0) return;
  if constexpr (KG == 1) lds_barrier();                          // nobody reads the buffers any more
  unsigned char *const dump = s_tiles + T::kParts + wave * dump_bytes(TN);
  switch (a.y_type) {
    case LUTKAN_F32: store_wave<LUTKAN_F32, TM, TN, GROUPED>(a, t, acc, row0, wave_col0, dump, scales); break;
    case LUTKAN_F16: store_wave<LUTKAN_F16, TM, TN, GROUPED>(a, t, acc, row0, wave_col0, dump, scales); break;
    default: store_wave<LUTKAN_BF16, TM, TN, GROUPED>(a, t, acc, row0, wave_col0, dump, scales); break;
  }
}

template <int TM, int TN, int WM, int WN, int KG, bool GROUPED, bool ASYNC>
int launch_tiles_as(ProductArgs a, int64_t row_tiles, const char *who, hipStream_t s) {
  using T = Tile<TM, TN, WM, WN, KG, ASYNC>;
  static LdsCap cap;
  a.extent = (int32_t)row_tiles;
  const auto kernel = lutkan_int8_tiled_kernel<TM, TN, WM, WN, KG, GROUPED, ASYNC>;
  if (int rc = raise_lds_cap(kernel, &cap, who)) return rc;
  lutkan::plan_note("int8_tiled rows=%d columns=%d teams=%d%s; ", T::kRows, T::kCols, KG, ASYNC ? " async" : "");
  hipLaunchKernelGGL(kernel, dim3((unsigned)(row_tiles * ((a.n + T::kCols - 1) / T::kCols))), dim3(T::kThreads * KG), T::kLds, s, a);
  return check_launch(who);
}

template <int TM, int TN, int WM, int WN, int KG, bool GROUPED>
int launch_tiles(const ProductArgs &a, int64_t row_tiles, bool async, const char *who, hipStream_t s) {
  return async ? launch_tiles_as<TM, TN, WM, WN, KG, GROUPED, true>(a, row_tiles, who, s) : launch_tiles_as<TM, TN, WM, WN, KG, GROUPED, false>(a, row_tiles, who, s);
}

// What a launch takes beyond an empty one (2.4 us in a replayed graph), in us, for the kernels' choice.  The constants were fitted to 650 drawn calls of 1 to
// 32768 rows, 16 to 8192 inputs and 2 to 8192 outputs, a third of them with rows at odd addresses, half by expert, each timed with every kernel; on 260 others the
// kernel that is taken was within 2 % of the quickest in 220, 1.02 times it in the geometric mean, 1.33 at worst (of all 910: 1.46, few steps of many tiles).  Tried beside these, and
// not worth their place: direct tiles of 32 x 32, four teams on 64 x 64, two on 128 x 128 (each is the quickest of 1 - 4 % of the calls, by little).
//   direct   what its work-groups read, each its own, over the whole GPU, and their number
//   tiled    rounds of as many tiles as fit the compute units, a tile's steps of 128 k: `one` where there is one to a compute unit, `all` where
//            there are `slots`, and `ends` before and behind the steps.  Where the number of tiles is a guess (groups) and two fit a compute
//            unit, a round that is begun counts by its part.
struct Call {
  const ProductArgs &a;
  bool grouped, aligned, async;
  double likely_tiles(int height) const {                        // of a routing of some spread: a group's last tile is half empty
    if (!grouped) return (double)(((int64_t)a.rows + height - 1) / height);
    const double some = (double)std::min(a.groups, a.rows), each = (double)a.rows / some;
    return some * std::max(1.0, each / height + (each > 1 ? 0.6 : 0.0));
  }
  double direct(int columns, double base, double rate, double by_expert, double times, double of_work_group) const {
    const double work_groups = likely_tiles(16) * ((a.n + columns - 1) / columns), rows = std::min(16.0, grouped ? (double)a.rows / std::min(a.groups, a.rows) : (double)a.rows);
    const double reads = work_groups * (rows + columns) * a.k / (rate * std::min(1.0, work_groups / 256));
    return base + reads * (aligned ? 1 : 1.6) * (grouped ? times : 1) + (grouped ? by_expert : 0) + of_work_group * std::max(0.0, work_groups - 512);      // (unaligned: five dwords for every four)
  }
  double tiled(int height, int width, int slots, int teams, double ends, double one, double all, double search, double end_block) const {
    const double tiles = likely_tiles(height) * ((a.n + width - 1) / width);
    const double steps = async ? a.k / 64 / 2.0 / teams : 2.0 * (a.k / 128) / teams;      // (through registers a step takes twice as long)
    ends += (grouped ? search : 0) + (a.k % (async ? 64 : 128) ? end_block : 0);
    if (grouped && slots > 1 && tiles > 256) return std::max(1.0, tiles / (256 * slots)) * (steps * all + ends);
    const double full = std::floor(tiles / (256 * slots)), rest = tiles - full * 256 * slots;
    return full * (steps * all + ends) + (rest > 0 ? steps * (rest <= 256 ? one : all) + ends : 0);
  }
};

template <bool GROUPED>
int launch_product(const ProductArgs &a, const char *who, hipStream_t s) {
  const auto tiles = [&](int height) {                           // no routing has more
    return GROUPED ? a.rows / height + (int64_t)std::min(a.groups + 1, a.rows) : ((int64_t)a.rows + height - 1) / height;
  };
  lutkan::plan_clear();
  const bool aligned = rows_aligned(a), async = aligned && copies_fit<GROUPED>(a);
  const Call call{a, GROUPED, aligned, async};
  enum { kDirect16x16, kDirect16x32, kTiled64, kTiled128, kTiled128x256, kTiled256, kKernels };
  double price[kKernels];
  price[kDirect16x16] = call.direct(16, 0.6, 9.8e6, 0.57, 1.58, 0.39e-3);
  price[kDirect16x32] = call.direct(32, 0.93, 11.6e6, 0.64, 1.44, 0.64e-3);
  price[kTiled64] = call.tiled(64, 64, 2, 2, 1.47, 0.416, 1.0, 1.0, 1.1);
  price[kTiled128] = call.tiled(128, 128, 2, 1, 2.54, 0.469, 1.31, 0.93, 2.2);
  price[kTiled128x256] = async ? call.tiled(128, 256, 2, 1, 4.6, 0.78, 2.43, 0.2, 1.8) : HUGE_VAL;      // (the sums of these two leave no registers to copy through)
  price[kTiled256] = async ? call.tiled(256, 256, 1, 1, 5.6, 1.17, 1.94, 0, 1.7) : HUGE_VAL;
  if (tiles(16) > 65535) price[kDirect16x16] = price[kDirect16x32] = HUGE_VAL;
  const auto beyond_a_launch = [&](int height, int width, int threads) { return !lutkan::launch_holds(tiles(height) * ((a.n + width - 1) / width), threads); };
  if (beyond_a_launch(64, 64, 512)) price[kTiled64] = HUGE_VAL;
  if (beyond_a_launch(128, 128, 256)) price[kTiled128] = HUGE_VAL;
  if (beyond_a_launch(128, 256, 256)) price[kTiled128x256] = HUGE_VAL;
  if (beyond_a_launch(256, 256, 512)) price[kTiled256] = HUGE_VAL;
  const int pick = (int)(std::min_element(price, price + kKernels) - price);
  if (price[pick] == HUGE_VAL) return fail(LUTKAN_EUNSUPPORTED, "%s: too many outputs", who);
  switch (pick) {
    case kDirect16x16: return launch_direct<1, 1, GROUPED>(a, tiles(16), aligned, who, s);
    case kDirect16x32: return launch_direct<1, 2, GROUPED>(a, tiles(16), aligned, who, s);
    case kTiled64: return launch_tiles<1, 1, 2, 2, 2, GROUPED>(a, tiles(64), async, who, s);
    case kTiled128x256: return launch_tiles_as<2, 4, 2, 2, 1, GROUPED, true>(a, tiles(128), who, s);
    case kTiled256: return launch_tiles_as<4, 2, 2, 4, 1, GROUPED, true>(a, tiles(256), who, s);
    default: return launch_tiles<2, 2, 2, 2, 1, GROUPED>(a, tiles(128), async, who, s);
  }
}

int check_product(const lutkan_matmul_fp8_args *p, const char *who, ProductArgs *a) {
  if (!p) return fail(LUTKAN_EINVAL, "%s: null arguments", who);
  if (p->rows < 0 || p->x_rows < 0 || p->k < 1 || p->n < 1) return fail(LUTKAN_EINVAL, "%s: rows %lld of %lld, %d x %d", who, (long long)p->rows, (long long)p->x_rows, p->n, p->k);
  if (p->k > LUTKAN_INT8_MAX_INPUTS) return fail(LUTKAN_EUNSUPPORTED, "%s: %d inputs, at most %d", who, p->k, LUTKAN_INT8_MAX_INPUTS);
  if (p->n > LUTKAN_FP8_MAX_INPUTS) return fail(LUTKAN_EUNSUPPORTED, "%s: %d outputs, at most %d", who, p->n, LUTKAN_FP8_MAX_INPUTS);
  if (!is_type(p->y_type)) return fail(LUTKAN_EINVAL, "%s: bad type", who);
  if (p->rows > 0 && (!p->x || !p->x_scales || !p->weight || !p->weight_scales || !p->y)) return fail(LUTKAN_EINVAL, "%s: null x / x_scales / weight / weight_scales / y", who);
  if (p->y_stride < p->n) return fail(LUTKAN_ESHAPE, "%s: a row of y is longer than its stride", who);
  if (p->x_stride < 0 || p->weight_stride < 0 || p->x_scales_stride < 0 || p->weight_matrix_stride < 0) return fail(LUTKAN_ESHAPE, "%s: negative stride", who);
  if (std::max({p->x_stride, p->weight_stride, p->x_scales_stride, p->y_stride, p->rows, p->x_rows}) > INT32_MAX)
    return fail(LUTKAN_EUNSUPPORTED, "%s: row strides and rows of at most 2^31 - 1", who);
  *a = ProductArgs{};
  a->x = static_cast<const unsigned char *>(p->x); a->w = static_cast<const unsigned char *>(p->weight);
  a->x_scales = p->x_scales; a->w_scales = p->weight_scales; a->y = static_cast<unsigned char *>(p->y);
  a->x_rows = (int32_t)p->x_rows; a->x_stride = (int32_t)p->x_stride; a->x_scales_stride = (int32_t)p->x_scales_stride;
  a->w_stride = (int32_t)p->weight_stride; a->w_matrix_stride = p->weight_matrix_stride; a->y_stride = (int32_t)p->y_stride;
  a->rows = (int32_t)p->rows; a->k = p->k; a->n = p->n; a->y_type = (int8_t)p->y_type;
  return LUTKAN_OK;
}

}  // namespace

extern "C" int lutkan_matmul_int8(const lutkan_matmul_fp8_args *p, void *hip_stream) {
  const char *who = "lutkan_matmul_int8";
  ProductArgs a;
  if (int rc = check_product(p, who, &a)) return rc;
  if (p->rows != p->x_rows) return fail(LUTKAN_ESHAPE, "%s: %lld rows out, %lld in", who, (long long)p->rows, (long long)p->x_rows);
  if (p->rows == 0) return LUTKAN_OK;
  return launch_product<false>(a, who, static_cast<hipStream_t>(hip_stream));
}

extern "C" int lutkan_grouped_matmul_int8(const lutkan_matmul_fp8_args *p, void *hip_stream) {
  const char *who = "lutkan_grouped_matmul_int8";
  ProductArgs a;
  if (int rc = check_product(p, who, &a)) return rc;
  if (p->groups < 1) return fail(LUTKAN_EINVAL, "%s: %d groups", who, p->groups);
  if (p->groups > LUTKAN_FP8_MAX_GROUPS) return fail(LUTKAN_EUNSUPPORTED, "%s: %d groups, at most %d", who, p->groups, LUTKAN_FP8_MAX_GROUPS);
  if (p->rows == 0) return LUTKAN_OK;
  if (!p->group_sizes) return fail(LUTKAN_EINVAL, "%s: null group_sizes", who);
  if ((p->group_sizes_bytes != 4 && p->group_sizes_bytes != 8) || (p->row_index && p->row_index_bytes != 4 && p->row_index_bytes != 8))
    return fail(LUTKAN_EINVAL, "%s: group_sizes and row_index are whole numbers of 4 or 8 bytes", who);
  if (p->rows > LUTKAN_FP8_MAX_GROUPED_ROWS) return fail(LUTKAN_EUNSUPPORTED, "%s: %lld rows, at most %d", who, (long long)p->rows, LUTKAN_FP8_MAX_GROUPED_ROWS);
  if (!p->row_index && p->rows != p->x_rows) return fail(LUTKAN_ESHAPE, "%s: %lld rows out, %lld in, and no row_index", who, (long long)p->rows, (long long)p->x_rows);
  if (p->row_index && p->x_rows == 0) return fail(LUTKAN_ESHAPE, "%s: row_index into no rows", who);
  a.group_sizes = p->group_sizes; a.row_index = p->row_index; a.groups = p->groups;
  a.group_sizes_bytes = (int8_t)p->group_sizes_bytes; a.row_index_bytes = (int8_t)p->row_index_bytes;
  return launch_product<true>(a, who, static_cast<hipStream_t>(hip_stream));
}
