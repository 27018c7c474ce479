// Products of 8-bit floating point codes (e4m3) with a scale for each block of 128 inputs:
//   y[s][n] = sum_b x_scale[s][b] * w_scale[n / 128][b] * sum_{k in block b} x[s][k] * w[n][k]
// for one weight, or for rows grouped by expert with a weight each.  A block's products are summed in the matrix core, the block's sum is
// multiplied by both scales and added in fp32.
//
// Which instruction: the one on 8-bit codes (16 x 16 x 128, a whole block) sums its products in groups of eight, in which it keeps 13
// bits below the leading bit of the largest and cuts off the rest (found with single products; all 8-bit forms do): 1.4e-5 of
// the result for normally distributed inputs, 1/100 of what the rounding to bf16 costs and 1/20 of that to f16.  Outputs of 16 bits are
// computed with it.  Outputs of 32 bits would lose by it what their type could hold, so for them every code is converted to bf16,
// which holds all of its values, and the product taken with the 16-bit instruction (16 x 16 x 32, four for a block, half the rate),
// whose sums are good to 2^-24.  Where a block's large products cancel, what the 8-bit instruction cuts is a part of them and not of their sum
// (at most 2^-10 of the sum of magnitudes): callers who need that ask for 32 bits.
//
// The weight is the instruction's first operand and the activations its second, so that a lane holds four neighbouring outputs of one
// row: one activation scale per lane, and outputs that are stored as a vector.  Both operands are read in the same order along k (a
// lane takes the 16-byte pieces p and p + 4 of a block's eight, p = lane / 16), so which k of the block the instruction takes first
// does not matter.
#include "lutkan_product.h"

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ i32x8 fragment(u32x4 low, u32x4 high) {
  return i32x8{(int)low.x, (int)low.y, (int)low.z, (int)low.w, (int)high.x, (int)high.y, (int)high.z, (int)high.w};
}

// A lane's 32 codes of a block as the instruction takes them: EXACT = false as they are, true as bf16.
template <bool EXACT>
struct Operand {
  i32x8 codes;
  __device__ __forceinline__ void set(i32x8 c) { codes = c; }
};
template <>
struct Operand<true> {
  bf16x8 value[4];
  __device__ __forceinline__ void set(i32x8 c) {
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const bf16x2 two = (e & 1) ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[e >> 1], 1.0f, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[e >> 1], 1.0f, false);
      value[e >> 2][2 * (e & 3)] = two[0];
      value[e >> 2][2 * (e & 3) + 1] = two[1];
    }
  }
};

__device__ __forceinline__ f32x4 block_product(const Operand<false> &w, const Operand<false> &x) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w.codes, x.codes, f32x4{0.0f, 0.0f, 0.0f, 0.0f}, 0, 0, 0, 0, 0, 0);   // both e4m3, no scales of its own
}
__device__ __forceinline__ f32x4 block_product(const Operand<true> &w, const Operand<true> &x) {
  f32x4 v{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int q = 0; q < 4; ++q) v = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w.value[q], x.value[q], v, 0, 0, 0);
  return v;
}

// Outputs that are not finite, once more.  Both scales meet before the block's sum: where their product passes fp32's range though each is
// finite, a sum of zero comes out as NaN and a small one as infinite.  Rows of the tile with such a block are computed again in
// fp64, an output to a lane, by the wave that stored them; other rows stay as they are.  (The kernels' loops have no place to look for
// it; this costs them one multiply-add an output.)
template <int ROWS, int COLS, bool GROUPED>
__device__ __forceinline__ void again_in_fp64(const RowTile &t, int64_t row0, int col0) {
  static_assert(kScaleBlock % COLS == 0, "columns of one block");
  uintptr_t args = (uintptr_t)__builtin_amdgcn_kernarg_segment_ptr();      // the arguments anew: kept until here they would take scalar registers throughout
  asm volatile("" : "+s"(args));
  const ProductArgs a = *reinterpret_cast<const ProductArgs *>(args);
  const int lane = threadIdx.x & 63, k_blocks = a.k_blocks();
  const float *ws = a.w_scales + ((int64_t)t.group * a.n_blocks() + col0 / kScaleBlock) * k_blocks;
  wait_all_vector_loads();                                       // (and stores: what is written here comes behind them)
#pragma unroll 1
  for (int part = 0; part < ROWS; part += 64) {
    bool beyond = false;
    const int64_t own = row0 + part + lane;
    if (part + lane < ROWS && own < t.end) {
      const int64_t from = source_row<GROUPED>(a, own);
      const float *xs = a.x_scales + max(from, (int64_t)0) * a.x_scales_stride;
      for (int b = 0; from >= 0 && b < k_blocks; ++b) beyond |= finite(xs[b]) && finite(ws[b]) && !finite(xs[b] * ws[b]);
    }
    for (unsigned long long rows = __ballot(beyond); rows != 0; rows &= rows - 1) {
      const int64_t row = row0 + part + __builtin_ctzll(rows), from = source_row<GROUPED>(a, row);
      const int col = col0 + lane;
      if (lane >= COLS || col >= a.n) continue;
      const unsigned char *x = a.x + from * a.x_stride, *w = a.w + t.group * a.w_matrix_stride + (int64_t)col * a.w_stride;
      const float *xs = a.x_scales + from * a.x_scales_stride;
      double sum = 0.0;
#pragma unroll 1
      for (int b = 0; b < k_blocks; ++b) {
        double of_block = 0.0;
#pragma unroll 1
        for (int k = b * kScaleBlock; k < min(a.k, (b + 1) * kScaleBlock); ++k)
          of_block += (double)(__builtin_amdgcn_cvt_f32_fp8(x[k], 0) * __builtin_amdgcn_cvt_f32_fp8(w[k], 0));
        sum += (double)xs[b] * (double)ws[b] * of_block;
      }
      unsigned char *to = a.y + (row * a.y_stride + col) * type_bytes(a.y_type);
      if (a.y_type == LUTKAN_F32) store_one<LUTKAN_F32>(to, (float)sum);
      else if (a.y_type == LUTKAN_F16) store_one<LUTKAN_F16>(to, (float)sum);
      else store_one<LUTKAN_BF16>(to, (float)sum);
    }
  }
}

// A work-group computes 16 MT rows x 16 NT columns from global memory straight into registers; its waves take the blocks of k in turn,
// and their sums meet in LDS in the waves' order.
// Bound by what it reads, as no work-group shares with another: 16 rows of 4096 -> 4096 7.2 us a call (16 x 16: 256 work-groups, one to a
// compute unit, weights 17 MB and as much of x again; 9.0 with 16 x 32); one row 5.3.
template <int MT, int NT, bool EXACT, bool GROUPED, bool ALIGNED>
__global__ __launch_bounds__(1024) void lutkan_fp8_direct_kernel(const ProductArgs a) {
  extern __shared__ __align__(16) f32x4 s_part[];                // [wave][row tile][column tile][lane]
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
  f32x4 acc[MT][NT];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[m][n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  bool none[MT];
  if (t.group >= 0) {
    const unsigned char *x[MT], *w[NT];
    const float *xs[MT], *ws = a.w_scales + ((int64_t)t.group * a.n_blocks() + col0 / kScaleBlock) * a.k_blocks();
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      const int64_t row = source_row<GROUPED>(a, min(t.first + 16 * m + (lane & 15), t.end - 1));
      none[m] = row < 0;
      x[m] = a.x + max(row, (int64_t)0) * a.x_stride;
      xs[m] = a.x_scales + max(row, (int64_t)0) * a.x_scales_stride;
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) w[n] = a.w + t.group * a.w_matrix_stride + (int64_t)min(col0 + 16 * n + (lane & 15), a.n - 1) * a.w_stride;
    // Codes and scales of a block, and its products: kDepth blocks are read before the first is multiplied.
    constexpr int kDepth = MT * NT == 1 ? 4 : MT * NT == 2 ? 2 : 1;
    struct Block { Piece<ALIGNED> w[NT][2], x[MT][2]; float scale[MT]; };
    const auto read_scales = [&](float (&scale)[MT], int b) {
#pragma unroll
      for (int m = 0; m < MT; ++m) scale[m] = xs[m][b] * ws[b];
    };
    const auto read = [&](Block &to, int b) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int n = 0; n < NT; ++n) to.w[n][h].read(w[n] + b * kScaleBlock + 64 * h + 16 * p);
#pragma unroll
        for (int m = 0; m < MT; ++m) to.x[m][h].read(x[m] + b * kScaleBlock + 64 * h + 16 * p);
      }
      read_scales(to.scale, b);
    };
    const auto multiply = [&](const i32x8 (&wc)[NT], const i32x8 (&xc)[MT], const float (&scale)[MT]) {
      Operand<EXACT> wf[NT], xf;
#pragma unroll
      for (int n = 0; n < NT; ++n) wf[n].set(wc[n]);
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        xf.set(xc[m]);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const f32x4 v = block_product(wf[n], xf);
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[m][n][e] = fmaf(scale[m], v[e], acc[m][n][e]);
        }
      }
    };
    const auto multiply_block = [&](const Block &of) {
      i32x8 wc[NT], xc[MT];
#pragma unroll
      for (int n = 0; n < NT; ++n) wc[n] = fragment(of.w[n][0].get(low_bits(w[n])), of.w[n][1].get(low_bits(w[n])));
#pragma unroll
      for (int m = 0; m < MT; ++m) xc[m] = fragment(of.x[m][0].get(low_bits(x[m])), of.x[m][1].get(low_bits(x[m])));
      multiply(wc, xc, of.scale);
    };
    const int whole = a.k / kScaleBlock;
    // The work-groups of an XCD begin at different blocks, so that they do not all ask for the same lines of x at a time (16 rows of
    // 4096 -> 4096 7.4 -> 7.2 us, 32 9.2 -> 9.1, one 5.6 -> 5.3).
    const int shift = whole ? (int)(blockIdx.x / 8 % (unsigned)whole) : 0;
    const auto turn = [&](int b) { return b + shift < whole ? b + shift : b + shift - whole; };
    for (int b = wave; b < whole; b += waves * kDepth) {
      Block held[kDepth];
#pragma unroll
      for (int d = 0; d < kDepth; ++d) if (b + d * waves < whole) read(held[d], turn(b + d * waves));
#pragma unroll
      for (int d = 0; d < kDepth; ++d) if (b + d * waves < whole) multiply_block(held[d]);
    }
    if (whole < a.k_blocks() && whole % waves == wave) {         // the last block, not whole
      i32x8 wc[NT], xc[MT];
      float scale[MT];
      const int k0 = whole * kScaleBlock + 16 * p;
#pragma unroll
      for (int n = 0; n < NT; ++n) wc[n] = fragment(piece_at_end(w[n], k0, a.k), piece_at_end(w[n], k0 + 64, a.k));
#pragma unroll
      for (int m = 0; m < MT; ++m) xc[m] = fragment(piece_at_end(x[m], k0, a.k), piece_at_end(x[m], k0 + 64, a.k));
      read_scales(scale, whole);
      multiply(wc, xc, scale);
    }
  } else {
#pragma unroll
    for (int m = 0; m < MT; ++m) none[m] = true;
  }
  if (waves > 1) {
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int n = 0; n < NT; ++n) s_part[((wave * MT + m) * NT + n) * 64 + lane] = acc[m][n];
    __syncthreads();
  }
  unsigned again = 0;                                            // tiles with outputs that are not finite
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      if ((m * NT + n) % waves != wave) continue;                // a wave sums every waves-th tile
      f32x4 v = acc[m][n];
      if (waves > 1) {
        v = s_part[(m * NT + n) * 64 + lane];
        for (int o = 1; o < waves; ++o) v += s_part[((o * MT + m) * NT + n) * 64 + lane];
      }
      if (none[m]) v = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      const int64_t row = t.first + 16 * m + (lane & 15);
      if (row < t.end) store_outputs(a, row, col0 + 16 * n + 4 * p, v);
      if (__any(!(finite(v.x) && finite(v.y) && finite(v.z) && finite(v.w)))) again |= 1u << (m * NT + n);
    }
  for (; again != 0; again &= again - 1) {
    const int tile = __builtin_ctz(again);
    again_in_fp64<16, 16, GROUPED>(t, t.first + 16 * (tile / NT), col0 + 16 * (tile % NT));
  }
}

template <int MT, int NT, bool EXACT, bool GROUPED>
int launch_direct(ProductArgs a, int64_t row_tiles, bool aligned, const char *who, hipStream_t s) {
  if (row_tiles > 65535) return fail(LUTKAN_EUNSUPPORTED, "%s: too many rows", who);
  const int waves = a.extent = std::min(a.k_blocks(), 16);
  const dim3 grid((unsigned)((a.n + 16 * NT - 1) / (16 * NT)), (unsigned)row_tiles);
  lutkan::plan_note("fp8_direct rows=%d columns=%d waves=%d; ", 16 * MT, 16 * NT, waves);
  const auto kernel = aligned ? lutkan_fp8_direct_kernel<MT, NT, EXACT, GROUPED, true> : lutkan_fp8_direct_kernel<MT, NT, EXACT, GROUPED, false>;
  hipLaunchKernelGGL(kernel, grid, dim3(64 * waves), waves > 1 ? (size_t)waves * MT * NT * 64 * sizeof(f32x4) : 0, s, a);
  return check_launch(who);
}

// A tile of 16 MT WM rows x 16 NT WN columns for a work-group of KG teams of WM x WN waves, each wave 16 MT rows x 16 NT columns of it.
// The teams take the blocks of k in turn; their sums meet in LDS in the teams' order.  A team's blocks (both operands' codes and their
// scales) go through LDS, in two buffers: while a block is multiplied the next is on its way.  A row's eight 16-byte pieces lie in an order that depends on the row (piece_place), so that the 16 rows that a read of 16 lanes takes
// lie in different banks (no conflict counted).
//   ASYNC: the pieces go from global memory to LDS without passing through registers: needs rows at dword addresses and
//   offsets that fit 32 bits.  Otherwise, and for a last block that is not whole, through registers.
// What it measured, into bf16, 8192 rows of 4096 -> 4096: 256 x 256 outputs 119 - 124 us on the same inputs again and again, 122 - 137 on three sets
// in turn (2.3 - 2.0 PFLOP/s; a library product of such codes with one scale for all 94), 128 x 128 157 and 189.  Matrix cores 0.46 busy: copies
// alone take 90 us, products and sums alone 105; codes of zeros 94 where random ones take 118, so that power decides too.  Into fp32
// (128 x 128) 259 and 273 - 281: every wave converts the codes that it reads, so each is converted twice, at half of the matrix rate (floor
// 173 - 187).  Teams, on the same inputs: 256 rows of the same 11.3 us with four on 64 x 64, 22 without; 128 x 128 18.6 with two, 26.5 without.
// The sizes of a tile, its buffers and its team.
template <int MT, int NT, int WM, int WN, int KG>
struct Tile {
  static constexpr int kRows = 16 * MT * WM, kCols = 16 * NT * WN, kThreads = 64 * WM * WN;
  static constexpr int kScalesAt = (kRows + kCols) * kScaleBlock, kStage = kScalesAt + (kRows + 4) * 4;      // codes, scales of the rows, of the columns' blocks
  static constexpr int kParts = KG > 1 ? (KG - 1) * kRows * kCols * 4 : 0;       // the sums of all teams but the one that adds them up
  static constexpr int kLds = KG * 2 * kStage > kParts ? KG * 2 * kStage : kParts;
  static_assert(kLds <= lutkan::kLdsPerWorkGroup && kStage % 16 == 0, "LDS");
};

template <int MT, int NT, int WM, int WN, int KG, bool EXACT, bool GROUPED, bool ASYNC>
__global__ __launch_bounds__(64 * WM * WN * KG, WM * WN * KG >= 16 ? 4 : 2) void lutkan_fp8_tiled_kernel(const ProductArgs a) {
  using T = Tile<MT, NT, WM, WN, KG>;
  constexpr int kRows = T::kRows, kCols = T::kCols, kWaves = WM * WN, kThreads = T::kThreads, kScalesAt = T::kScalesAt, kStage = T::kStage;
  constexpr int kXCopies = kRows / 8 / kWaves, kWCopies = kCols / 8 / kWaves, kCopies = kXCopies + kWCopies;     // of 8 rows, for each wave
  static_assert(kXCopies * 8 * kWaves == kRows && kWCopies * 8 * kWaves == kCols && kXCopies % 2 == 0 && kWCopies % 2 == 0, "copies in pairs");
  static_assert(kThreads >= kRows && kScaleBlock % (16 * NT) == 0, "tile");
  extern __shared__ __align__(16) unsigned char s_tiles[];       // [team][buffer][rows of x, rows of the weight][128], scales
  const int lane = threadIdx.x & 63, wave_of_all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), team = wave_of_all / kWaves;
  const int wave = wave_of_all % kWaves, tid = wave * 64 + lane, wm = wave / WN, wn = wave % WN, p = lane >> 4;
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
  f32x4 acc[MT][NT];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[m][n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  if (t.group >= 0) {
    const unsigned char *w_tile = a.w + t.group * a.w_matrix_stride + (int64_t)col0 * a.w_stride;
    const unsigned char *x_tile = GROUPED ? a.x : a.x + t.first * a.x_stride;
    const float *scales_tile = GROUPED ? a.x_scales : a.x_scales + t.first * a.x_scales_stride;
    typedef std::conditional_t<ASYNC, unsigned, int64_t> offset_t;
    offset_t x_from[kXCopies], w_from[kWCopies], scale_from;     // the rows that this lane's pieces, and its scale, come from
    int piece_at[2];                                             // and the columns: place i of row r, the same for every 16 rows
#pragma unroll
    for (int c = 0; c < 2; ++c) piece_at[c] = piece_place(c * 8 + (lane >> 3), lane & 7) * 16;        // (its own inverse)
    const auto row_of = [&](int r) {                             // rows behind the last are the last again
      const int64_t row = min(t.first + r, t.end - 1);
      return GROUPED ? max(source_row<GROUPED>(a, row), (int64_t)0) : row - t.first;
    };
#pragma unroll
    for (int c = 0; c < kXCopies; ++c) x_from[c] = (offset_t)(row_of((wave * kXCopies + c) * 8 + (lane >> 3)) * a.x_stride);
#pragma unroll
    for (int c = 0; c < kWCopies; ++c) w_from[c] = (offset_t)((int64_t)min((wave * kWCopies + c) * 8 + (lane >> 3), a.n - 1 - col0) * a.w_stride);
    scale_from = (offset_t)(row_of(min(tid, kRows - 1)) * a.x_scales_stride * 4);
    constexpr int kColBlocks = kCols > kScaleBlock ? kCols / kScaleBlock : 1;    // (a tile of fewer columns lies in one block)
    const float *w_scales_tile = a.w_scales + ((int64_t)t.group * a.n_blocks() + col0 / kScaleBlock) * a.k_blocks();
    const unsigned w_scale_from = (unsigned)(min(lane, a.n_blocks() - 1 - col0 / kScaleBlock) * a.k_blocks()) * 4;
    const int whole = a.k / kScaleBlock, own = (whole - team + KG - 1) / KG, steps = (whole + KG - 1) / KG;     // whole blocks: all, this team's, the first team's
    unsigned char *const s_team = s_tiles + team * 2 * kStage;
    const auto block_of = [&](int step) { return step * KG + team; };
    const auto stage = [&](int step) { return s_team + (step & 1) * kStage; };
    Piece<false> held[ASYNC ? 1 : kCopies];                      // (without ASYNC: rows at any address)
    float held_scale, held_w_scale;
    const auto ask_scales = [&](int64_t b) {
      held_scale = load_any<float>(reinterpret_cast<const unsigned char *>(scales_tile + b) + scale_from);
      held_w_scale = load_any<float>(reinterpret_cast<const unsigned char *>(w_scales_tile + b) + w_scale_from);
    };
    // The pieces of this team's block of a step are asked for, copy by copy, and put into their buffer: at once where they go straight
    // there, else by put().
    const auto ask = [&](int step, int c) {
      const bool of_x = c < kXCopies;
      const int cw = c - kXCopies;
      const int64_t b = block_of(step);
      if constexpr (ASYNC) {
        unsigned char *to = stage(step) + (of_x ? (wave * kXCopies + c) * 1024 : kRows * kScaleBlock + (wave * kWCopies + cw) * 1024);
        copy16_global_to_lds_at((of_x ? x_tile : w_tile) + b * kScaleBlock, (of_x ? x_from[c] : w_from[cw]) + piece_at[c & 1], to);
        if (c == 0 && wave < kRows / 64) copy4_global_to_lds_at(scales_tile + b, scale_from, stage(step) + kScalesAt + wave * 256);
        if (c == 0 && wave == kWaves - 1 && lane < kColBlocks) copy4_global_to_lds_at(w_scales_tile + b, w_scale_from, stage(step) + kScalesAt + kRows * 4);
      } else {
        if (c == 0) ask_scales(b);
        held[c].read((of_x ? x_tile + x_from[c] : w_tile + w_from[cw]) + (b * kScaleBlock + piece_at[c & 1]));
      }
    };
    const auto put_scales = [&](int step) {
      float *to = reinterpret_cast<float *>(stage(step) + kScalesAt);
      if (tid < kRows) to[tid] = held_scale;
      if (tid < kColBlocks) to[kRows + tid] = held_w_scale;
    };
    const auto put = [&](int step) {
      if constexpr (!ASYNC) {
        unsigned char *to = stage(step) + lane * 16;
#pragma unroll
        for (int c = 0; c < kXCopies; ++c) *reinterpret_cast<u32x4 *>(to + (wave * kXCopies + c) * 1024) = held[c].get(low_bits(x_tile + x_from[c]));
#pragma unroll
        for (int c = 0; c < kWCopies; ++c) *reinterpret_cast<u32x4 *>(to + kRows * kScaleBlock + (wave * kWCopies + c) * 1024) = held[kXCopies + c].get(low_bits(w_tile + w_from[c]));
        put_scales(step);
      }
    };
    // The last block, if it is not whole: this team's step `own`.
    const auto put_end = [&]() {
      ask_scales(whole);
      unsigned char *to = stage(own) + lane * 16;
      for (int c = 0; c < kXCopies; ++c)
        *reinterpret_cast<u32x4 *>(to + (wave * kXCopies + c) * 1024) = piece_at_end(x_tile + x_from[c], whole * kScaleBlock + piece_at[c & 1], a.k);
      for (int c = 0; c < kWCopies; ++c)
        *reinterpret_cast<u32x4 *>(to + kRows * kScaleBlock + (wave * kWCopies + c) * 1024) = piece_at_end(w_tile + w_from[c], whole * kScaleBlock + piece_at[c & 1], a.k);
      put_scales(own);
    };
    const int at_row = lane & 15, low = at_row * kScaleBlock + piece_place(at_row, p) * 16, high_half = at_row * kScaleBlock + piece_place(at_row, p + 4) * 16;
    // One block: the products in a fixed order, each added two products after it was begun; a row subtile's codes are read while the one
    // before it is multiplied.
    const auto multiply = [&](int step, bool ask_next) {
      const unsigned char *xt = stage(step) + (wm * 16 * MT) * kScaleBlock;
      const unsigned char *wt = stage(step) + (kRows + wn * 16 * NT) * kScaleBlock;
      const float *scales = reinterpret_cast<const float *>(stage(step) + kScalesAt) + wm * 16 * MT + at_row;
      const float w_scale = scales[kRows + wn * 16 * NT / kScaleBlock - (wm * 16 * MT + at_row)];
      const auto codes = [&](const unsigned char *rows, int sub) {
        return fragment(*reinterpret_cast<const u32x4 *>(rows + sub * 16 * kScaleBlock + low), *reinterpret_cast<const u32x4 *>(rows + sub * 16 * kScaleBlock + high_half));
      };
      i32x8 next = codes(xt, 0), wc[NT];
      float next_scale = scales[0];
#pragma unroll
      for (int n = 0; n < NT; ++n) {                             // in the order of their first products
        wc[n] = codes(wt, n);
        __builtin_amdgcn_sched_barrier(0);
      }
      Operand<EXACT> wf[NT];
      Operand<EXACT> xf;
      constexpr int kAhead = 2, kEvery = MT * NT / kCopies >= 2 ? 2 : 1;
      static_assert(kEvery * kCopies <= MT * NT, "copies");
      f32x4 v[kAhead + 1];
      float scales_of[2];
#pragma unroll
      for (int i = 0; i < MT * NT + kAhead; ++i) {
        const int m = i / NT, n = i % NT;
        if (i < MT * NT) {
          if (n == 0) {
            xf.set(next);
            scales_of[m & 1] = next_scale * w_scale;
            if (m + 1 < MT) {
              next = codes(xt, m + 1);
              next_scale = scales[(m + 1) * 16];
            }
          }
          if (m == 0) wf[n].set(wc[n]);
          v[i % (kAhead + 1)] = block_product(wf[n], xf);
          __builtin_amdgcn_sched_barrier(0);
          // Copies in between: a wave waits for its turn with each, and all at once would keep it from its products.
          if (i % kEvery == kEvery - 1 && i / kEvery < kCopies && ask_next) ask(step + 1, i / kEvery);
        }
        if (i >= kAhead) {
          const int of = i - kAhead;
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[of / NT][of % NT][e] = fmaf(scales_of[(of / NT) & 1], v[of % (kAhead + 1)][e], acc[of / NT][of % NT][e]);
          asm volatile("" : "+v"(acc[of / NT][of % NT]));        // (here, not behind the next branch, with all products held until then)
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    if (own > 0) {
#pragma unroll
      for (int c = 0; c < kCopies; ++c) ask(0, c);
      put(0);
    }
    for (int step = 0; step < steps; ++step) {
      wait_all_vector_loads();
      lds_barrier();                                             // the block is there, and nobody reads the buffer of the one before it any more
      if (step < own) multiply(step, step + 1 < own);
      if (step + 1 < own) put(step + 1);
    }
    if (whole < a.k_blocks()) {
      const bool mine = whole % KG == team;
      if (mine) put_end();                                       // (into a buffer that nobody reads since the last barrier)
      lds_barrier();
      if (mine) multiply(own, false);
    }
    if constexpr (KG > 1) {
      lds_barrier();                                             // nobody reads the buffers any more
      f32x4 *parts = reinterpret_cast<f32x4 *>(s_tiles);         // [team - 1][wave][m][n][lane]
      if (team > 0) {
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int n = 0; n < NT; ++n) parts[((((team - 1) * kWaves + wave) * MT + m) * NT + n) * 64 + lane] = acc[m][n];
      }
      lds_barrier();
      if (team > 0) return;
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int n = 0; n < NT; ++n)
          for (int o = 0; o < KG - 1; ++o) acc[m][n] += parts[(((o * kWaves + wave) * MT + m) * NT + n) * 64 + lane];
    }
  }
  if (KG > 1 && team > 0) return;
  f32x4 seen{0.0f, 0.0f, 0.0f, 0.0f};                            // NaN once an output is not finite
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    const int64_t row = t.first + (wm * MT + m) * 16 + (lane & 15);
    const bool none = t.group < 0 || (GROUPED && row < t.end && source_row<GROUPED>(a, row) < 0);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      acc[m][n] = none ? f32x4{0.0f, 0.0f, 0.0f, 0.0f} : acc[m][n];
#pragma unroll
      for (int e = 0; e < 4; ++e) seen[e] = fmaf(acc[m][n][e], 0.0f, seen[e]);
    }
    store_row<NT>(a, row, row < t.end, col0 + wn * NT * 16, p, acc[m]);
  }
  if (__any((seen[0] + seen[1]) + (seen[2] + seen[3]) != 0.0f)) again_in_fp64<16 * MT, 16 * NT, GROUPED>(t, t.first + wm * MT * 16, col0 + wn * NT * 16);
}

template <int MT, int NT, int WM, int WN, int KG, bool EXACT, bool GROUPED, bool ASYNC>
int launch_tiles_as(ProductArgs a, int64_t row_tiles, const char *who, hipStream_t s) {
  using T = Tile<MT, NT, WM, WN, KG>;
  static LdsCap cap;
  a.extent = (int32_t)row_tiles;
  const auto kernel = lutkan_fp8_tiled_kernel<MT, NT, WM, WN, KG, EXACT, GROUPED, ASYNC>;
  if (int rc = raise_lds_cap(kernel, &cap, who)) return rc;
  lutkan::plan_note("fp8_tiled rows=%d columns=%d teams=%d%s; ", T::kRows, T::kCols, KG, ASYNC ? " async" : "");
  hipLaunchKernelGGL(kernel, dim3((unsigned)(row_tiles * ((a.n + T::kCols - 1) / T::kCols))), dim3(T::kThreads * KG), T::kLds, s, a);
  return check_launch(who);
}

template <int MT, int NT, int WM, int WN, int KG, bool EXACT, bool GROUPED>
int launch_tiles(const ProductArgs &a, int64_t row_tiles, bool async, const char *who, hipStream_t s) {
  return async ? launch_tiles_as<MT, NT, WM, WN, KG, EXACT, GROUPED, true>(a, row_tiles, who, s) : launch_tiles_as<MT, NT, WM, WN, KG, EXACT, GROUPED, false>(a, row_tiles, who, s);
}

// What a launch takes beyond an empty one, in us, for the kernels' choice; the constants were fitted to times from 1 to 8192 rows, 128 to 8192
// inputs and 256 to 8192 outputs.  The prices order the kernels; as times they are rough: with 2.4 us for the launch 0.84 of the
// measured time in the median of 160 drawn calls, 0.54 - 1.13 for nine of ten, 0.3 at worst (few inputs, ragged groups).  On 140 other
// drawn calls, each timed with every kernel that was not hopeless, the one that is taken was within 2 % of the quickest in 110,
// 1.03 times it in the geometric mean, 1.45 at worst.
//   direct   what its work-groups read, each its own: 9 MB/us over the whole GPU
//   tiled    rounds of as many tiles as fit the compute units, a tile's steps over k: `one` where there is one to a compute unit, `all` where
//            there are `slots`, and `ends` before and behind the steps.  Where the number of tiles is a guess (groups) and two fit a compute
//            unit, a round that is begun counts by its part.  (Too little for long ragged groups: 16384 rows of 2048 -> 1024 in 32 groups are priced
//            44 with 128 x 128 and 63 with 256 x 256, and take 79 and 78; in even groups 64 and 45.)
// What the choice is worth, us: 16 rows of 4096 -> 4096 7.2 with 16 x 16, 9.0 with 16 x 32; 256 of them 11.3 with four teams on 64 x 64, 11.6 with two, 26.5
// with 128 x 128; 614 of 6472 -> 3900 49 with two teams on 128 x 128, 60 with one, 65 with two on 64 x 64 (into fp32 5076 of 7936 -> 711 64, 95, 83).
// (All on the same inputs again and again.)
inline double direct_price(double row_tiles, double rows_of_tile, int columns, const ProductArgs &a) {
  const double work_groups = row_tiles * ((a.n + columns - 1) / columns);
  return work_groups * (rows_of_tile + columns) * a.k / (9e6 * std::min(1.0, work_groups / 256));
}
inline double tiled_price(double tiles, int slots, double one, double all, double ends, double steps, bool guess) {
  if (guess && slots > 1 && tiles > 256) return std::max(1.0, tiles / (256 * slots)) * (steps * all + ends);
  const double full = std::floor(tiles / (256 * slots)), rest = tiles - full * 256 * slots;
  return full * (steps * all + ends) + (rest > 0 ? steps * (rest <= 256 ? one : all) + ends : 0);
}

template <bool EXACT, bool GROUPED>
int launch_product(const ProductArgs &a, const char *who, hipStream_t s) {
  const int64_t groups = GROUPED ? a.groups : 1;
  const auto tiles = [&](int height) {                           // no routing has more
    return GROUPED ? a.rows / height + std::min<int64_t>(groups + 1, a.rows) : ((int64_t)a.rows + height - 1) / height;
  };
  const auto likely_tiles = [&](int height) {                    // of a routing of some spread: a group's last tile is half empty
    if (!GROUPED) return (double)tiles(height);
    const double some = (double)std::min<int64_t>(groups, a.rows), each = (double)a.rows / some;
    return some * std::max(1.0, each / height + (each > 1 ? 0.6 : 0.0));
  };
  lutkan::plan_clear();
  const bool aligned = rows_aligned(a), async = aligned && copies_fit<GROUPED>(a);
  const double likely_rows = (double)a.rows / (double)std::min<int64_t>(groups, a.rows);
  const double end_block = a.k % kScaleBlock ? 2.5 : 0;          // (read, put and multiplied behind the others)
  const auto tiled = [&](int side, int slots, double one, double all, double ends, int teams) {
    // Through registers a step waits longer.  Into 16 bits the step has the factor: with those of 32 bits, 12 of 120 drawn calls took other kernels, and
    // what they take now is 0.81 of that (0.59 - 1.37 each); into 32 bits a factor for the step did not pay (1.10).
    const double step = async || EXACT ? 1 : side == 64 ? 1.75 : 1.5;
    return tiled_price(likely_tiles(side) * ((a.n + side - 1) / side), slots, one * step, all * step, ends + end_block, std::ceil(a.k / kScaleBlock / (double)teams), GROUPED);
  };
  enum { kDirect16x16, kDirect16x32, kDirect32x32, kTiled64x4, kTiled64x2, kTiled128x2, kTiled128, kTiled256, kKernels };
  double price[kKernels];
  price[kDirect16x16] = direct_price(likely_tiles(16), std::min(16.0, likely_rows), 16, a);
  price[kDirect16x32] = direct_price(likely_tiles(16), std::min(16.0, likely_rows), 32, a);
  price[kDirect32x32] = direct_price(likely_tiles(32), std::min(32.0, likely_rows), 32, a);
  constexpr double kSearch = GROUPED ? 2 : 0;                    // for the group, before a small tile's few steps
  price[kTiled64x4] = EXACT ? tiled(64, 1, 1.05, 1.4, 1 + kSearch, 4) : tiled(64, 1, 0.62, 1.0, 1 + kSearch, 4);
  price[kTiled64x2] = EXACT ? tiled(64, 2, 0.62, 1.3, 1 + kSearch, 2) : tiled(64, 2, 0.36, 0.85, 1 + kSearch, 2);
  price[kTiled128x2] = EXACT ? tiled(128, 1, 1.75, 1.75, 5, 2) : tiled(128, 1, 1.0, 1.0, 5, 2);
  price[kTiled128] = EXACT ? tiled(128, 2, 1.3, 1.9, 2, 1) : tiled(128, 2, 0.65, 1.08, 2, 1);
  price[kTiled256] = EXACT ? HUGE_VAL : tiled(256, 1, 1.6, 1.6, 6, 1);
  if (GROUPED)                                                   // (weights that few rows share come from memory)
    for (int k = kDirect16x16; k <= kDirect32x32; ++k) price[k] *= 1.7;
  if (!aligned)                                                  // (five dwords for every four)
    for (int k = kDirect16x16; k <= kDirect32x32; ++k) price[k] *= EXACT ? 1.6 : 2;
  if (!async) price[kTiled256] = HUGE_VAL;                       // (its sums leave no registers to copy through)
  if (!async && EXACT) {
    // Through registers: steps and ends in one.  The factors carry spilled registers too: a piece that is held takes five, beside fragments of
    // bf16, and all of these but 64 x 64 with two teams spill 12 - 30 (52 - 92 bytes a lane).
    price[kTiled64x4] *= 2, price[kTiled64x2] *= 2;
    price[kTiled128x2] *= 1.5, price[kTiled128] *= 1.5;
  }
  if (tiles(16) > 65535) price[kDirect16x16] = price[kDirect16x32] = HUGE_VAL;
  if (tiles(32) > 65535) price[kDirect32x32] = HUGE_VAL;
  const auto beyond_a_launch = [&](int side, int threads) { return !lutkan::launch_holds(tiles(side) * ((a.n + side - 1) / side), threads); };
  if (beyond_a_launch(64, 1024)) price[kTiled64x4] = HUGE_VAL;
  if (beyond_a_launch(64, 512)) price[kTiled64x2] = HUGE_VAL;
  if (beyond_a_launch(128, 512)) price[kTiled128x2] = HUGE_VAL;
  if (beyond_a_launch(128, 256)) price[kTiled128] = HUGE_VAL;
  if (beyond_a_launch(256, 512)) price[kTiled256] = HUGE_VAL;
  const int pick = (int)(std::min_element(price, price + kKernels) - price);
  if (price[pick] == HUGE_VAL) return fail(LUTKAN_EUNSUPPORTED, "%s: too many outputs", who);
  switch (pick) {
    case kDirect16x16: return launch_direct<1, 1, EXACT, GROUPED>(a, tiles(16), aligned, who, s);
    case kDirect16x32: return launch_direct<1, 2, EXACT, GROUPED>(a, tiles(16), aligned, who, s);
    case kDirect32x32: return launch_direct<2, 2, EXACT, GROUPED>(a, tiles(32), aligned, who, s);
    case kTiled64x4: return launch_tiles<2, 2, 2, 2, 4, EXACT, GROUPED>(a, tiles(64), async, who, s);
    case kTiled64x2: return launch_tiles<2, 2, 2, 2, 2, EXACT, GROUPED>(a, tiles(64), async, who, s);
    case kTiled128x2: return launch_tiles<4, 4, 2, 2, 2, EXACT, GROUPED>(a, tiles(128), async, who, s);
    case kTiled256: if constexpr (!EXACT) return launch_tiles_as<8, 4, 2, 4, 1, EXACT, GROUPED, true>(a, tiles(256), who, s);
    default: return launch_tiles<4, 4, 2, 2, 1, EXACT, GROUPED>(a, tiles(128), async, who, s);
  }
}

int check_product(const lutkan_matmul_fp8_args *p, const char *who, ProductArgs *a) {
  if (!p) return fail(LUTKAN_EINVAL, "%s: null arguments", who);
  if (p->rows < 0 || p->x_rows < 0 || p->k < 1 || p->n < 1) return fail(LUTKAN_EINVAL, "%s: rows %lld of %lld, %d x %d", who, (long long)p->rows, (long long)p->x_rows, p->n, p->k);
  if (p->k > LUTKAN_FP8_MAX_INPUTS) return fail(LUTKAN_EUNSUPPORTED, "%s: %d inputs, at most %d", who, p->k, LUTKAN_FP8_MAX_INPUTS);
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

extern "C" int lutkan_matmul_fp8(const lutkan_matmul_fp8_args *p, void *hip_stream) {
  const char *who = "lutkan_matmul_fp8";
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  ProductArgs a;
  if (int rc = check_product(p, who, &a)) return rc;
  if (p->rows != p->x_rows) return fail(LUTKAN_ESHAPE, "%s: %lld rows out, %lld in", who, (long long)p->rows, (long long)p->x_rows);
  if (p->rows == 0) return LUTKAN_OK;
  return a.y_type == LUTKAN_F32 ? launch_product<true, false>(a, who, s) : launch_product<false, false>(a, who, s);
}

extern "C" int lutkan_grouped_matmul_fp8(const lutkan_matmul_fp8_args *p, void *hip_stream) {
  const char *who = "lutkan_grouped_matmul_fp8";
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
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
  return a.y_type == LUTKAN_F32 ? launch_product<true, true>(a, who, s) : launch_product<false, true>(a, who, s);
}
