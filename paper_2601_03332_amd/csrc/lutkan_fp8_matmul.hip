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
// whose sums are good to 2^-24.
//
// The weight is the instruction's first operand and the activations its second, so that a lane holds four neighbouring outputs of one
// row: one activation scale per lane, and outputs that are stored as a vector.  Both operands are read in the same order along k (a
// lane takes the 16-byte pieces p and p + 4 of a block's eight, p = lane / 16), so which k of the block the instruction takes first
// does not matter.
#include "lutkan_fp8.h"

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

struct ProductArgs {
  const unsigned char *x, *w;
  const float *x_scales, *w_scales;
  unsigned char *y;
  int64_t x_rows, x_stride, x_scales_stride, w_stride, w_matrix_stride, y_stride;    // bytes of codes, elements of scales and outputs
  int64_t rows;
  int32_t k, n, k_blocks, n_blocks, y_type;
  const void *group_sizes, *row_index;
  int32_t groups, group_sizes_bytes, row_index_bytes;
};

__device__ __forceinline__ i32x8 fragment(u32x4 low, u32x4 high) {
  return i32x8{(int)low.x, (int)low.y, (int)low.z, (int)low.w, (int)high.x, (int)high.y, (int)high.z, (int)high.w};
}

// Sixteen codes of a row from column k0 on, zeros beyond its end; no byte behind the row is read.
__device__ u32x4 piece_at_end(const unsigned char *row, int k0, int k) {
  if (k0 + 16 <= k) return load_any<u32x4>(row + k0);
  u32x4 v{0, 0, 0, 0};
  if (k0 >= k) return v;
  if (k >= 16) {                                                 // the row's last sixteen, moved down
    const unsigned __int128 last = load_any<unsigned __int128>(row + k - 16) >> (8 * (k0 + 16 - k));
    return __builtin_bit_cast(u32x4, last);
  }
  unsigned __int128 codes = 0;
  for (int e = k - k0 - 1; e >= 0; --e) codes = (codes << 8) | row[k0 + e];
  return __builtin_bit_cast(u32x4, codes);
}

// The 32 codes of a block that lane-sixteenth `p` takes of a row.
template <bool END>
__device__ __forceinline__ i32x8 block_of_row(const unsigned char *row, int k0, int p, int k) {
  if constexpr (END) return fragment(piece_at_end(row, k0 + 16 * p, k), piece_at_end(row, k0 + 64 + 16 * p, k));
  else return fragment(load_any<u32x4>(row + k0 + 16 * p), load_any<u32x4>(row + k0 + 64 + 16 * p));
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

// Four neighbouring outputs of a row, those that exist.
__device__ __forceinline__ void store_outputs(const ProductArgs &a, int64_t row, int col, f32x4 v) {
  if (col >= a.n) return;
  if (a.y_type == LUTKAN_F32) {
    unsigned char *p = a.y + (row * a.y_stride + col) * 4;
    if (col + 4 <= a.n) { store_any(p, v); return; }
    for (int e = 0; e < 4; ++e) if (col + e < a.n) store_any(p + 4 * e, v[e]);
    return;
  }
  unsigned char *p = a.y + (row * a.y_stride + col) * 2;
  unsigned bits[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) bits[e] = a.y_type == LUTKAN_F16 ? f16_bits(v[e]) : bf16_bits(v[e]);
  if (col + 4 <= a.n) { store_any(p, u32x2{bits[0] | (bits[1] << 16), bits[2] | (bits[3] << 16)}); return; }
#pragma unroll
  for (int e = 0; e < 4; ++e) if (col + e < a.n) store_any(p + 2 * e, (unsigned short)bits[e]);
}

// Rows [first, end) of the tile, of one group; group < 0: rows behind the last group, whose outputs are zeros.  end <= first: none.
struct RowTile { int64_t first, end; int group; };

// Tile `tile` of the rows, cut at the groups' ends: every group's rows in tiles of `height`, then those behind the last group.  The
// sizes are the caller's, on the device: negative ones count as none, and a group ends with the rows at the latest.  Each wave for
// itself, a lane a group, 64 groups at a time.  `first_behind`: the first tile behind the last group.
__device__ __forceinline__ RowTile grouped_tile(const ProductArgs &a, int64_t tile, int height, int64_t *first_behind = nullptr) {
  const int lane = threadIdx.x & 63;
  int64_t row0 = 0, tile0 = 0;
  for (int base = 0; base < a.groups; base += 64) {
    int64_t size = 0;
    if (base + lane < a.groups) size = a.group_sizes_bytes == 8 ? static_cast<const int64_t *>(a.group_sizes)[base + lane] : static_cast<const int32_t *>(a.group_sizes)[base + lane];
    size = size < 0 ? 0 : size > a.rows ? a.rows : size;
    int64_t end = size;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const int64_t below = __shfl_up(end, off);
      if (lane >= off) end += below;
    }
    const int64_t first = min(row0 + end - size, a.rows);
    end = min(row0 + end, a.rows);
    const int64_t own = (end - first + height - 1) / height;
    int64_t last_tile = own;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const int64_t below = __shfl_up(last_tile, off);
      if (lane >= off) last_tile += below;
    }
    last_tile += tile0;
    const unsigned long long here = __ballot(tile < last_tile);
    if (here != 0) {
      const int owner = __builtin_amdgcn_readfirstlane(__builtin_ctzll(here));
      const int64_t at = __shfl(first, owner) + (tile - (__shfl(last_tile, owner) - __shfl(own, owner))) * height;
      return {at, min(at + height, __shfl(end, owner)), base + owner};
    }
    row0 = __shfl(end, 63);
    tile0 = __shfl(last_tile, 63);
  }
  if (first_behind) *first_behind = tile0;
  const int64_t at = row0 + (tile - tile0) * height;
  return {at, min(at + height, a.rows), -1};
}

// A value that every lane of the wave holds, as one.
__device__ __forceinline__ int64_t uniform(int64_t v) {
  return ((int64_t)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32) | (unsigned)__builtin_amdgcn_readfirstlane((int)v);
}

// All tiles of the rows, those behind the last group among them.
__device__ __forceinline__ int64_t grouped_tiles(const ProductArgs &a, int height) {
  constexpr int64_t kBeyond = (int64_t)1 << 62;
  int64_t tiles = 0;
  const RowTile none = grouped_tile(a, kBeyond / height, height, &tiles);
  const int64_t rest = a.rows - (none.first - (kBeyond / height - tiles) * height);
  return tiles + (rest + height - 1) / height;
}

// The row of x behind row `row` of the outputs; -1: none, a row of zeros.
template <bool GROUPED>
__device__ __forceinline__ int64_t source_row(const ProductArgs &a, int64_t row) {
  if constexpr (GROUPED) {
    if (a.row_index) {
      const int64_t r = a.row_index_bytes == 8 ? static_cast<const int64_t *>(a.row_index)[row] : static_cast<const int32_t *>(a.row_index)[row];
      return r >= 0 && r < a.x_rows ? r : -1;
    }
  }
  return row;
}

// A work-group computes 16 MT rows x 16 NT columns from global memory straight into registers; its waves take the blocks of k in turn,
// and their sums meet in LDS in the waves' order.
template <int MT, int NT, bool EXACT, bool GROUPED>
__global__ __launch_bounds__(MT * NT == 1 ? 1024 : 512) void lutkan_fp8_direct_kernel(const ProductArgs a) {
  extern __shared__ __align__(16) f32x4 s_part[];                // [wave][row tile][column tile][lane]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  const int p = lane >> 4, col0 = blockIdx.x * (16 * NT);
  RowTile t;
  if constexpr (GROUPED) {
    t = grouped_tile(a, blockIdx.y, 16 * MT);
    if (t.end <= t.first) return;
  } else {
    t.first = (int64_t)blockIdx.y * (16 * MT);
    t.end = min(t.first + 16 * MT, a.rows);
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
    const float *xs[MT], *ws = a.w_scales + ((int64_t)t.group * a.n_blocks + col0 / kScaleBlock) * a.k_blocks;
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      const int64_t row = source_row<GROUPED>(a, min(t.first + 16 * m + (lane & 15), t.end - 1));
      none[m] = row < 0;
      x[m] = a.x + max(row, (int64_t)0) * a.x_stride;
      xs[m] = a.x_scales + max(row, (int64_t)0) * a.x_scales_stride;
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) w[n] = a.w + t.group * a.w_matrix_stride + (int64_t)min(col0 + 16 * n + (lane & 15), a.n - 1) * a.w_stride;
    const auto block = [&](int b, auto at_end) {
      i32x8 wc[NT], xc[MT];
#pragma unroll
      for (int n = 0; n < NT; ++n) wc[n] = block_of_row<decltype(at_end)::value>(w[n], b * kScaleBlock, p, a.k);
#pragma unroll
      for (int m = 0; m < MT; ++m) xc[m] = block_of_row<decltype(at_end)::value>(x[m], b * kScaleBlock, p, a.k);
      Operand<EXACT> wf[NT], xf;
#pragma unroll
      for (int n = 0; n < NT; ++n) wf[n].set(wc[n]);
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        const float scale = xs[m][b] * ws[b];
        xf.set(xc[m]);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const f32x4 v = block_product(wf[n], xf);
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[m][n][e] = fmaf(scale, v[e], acc[m][n][e]);
        }
      }
    };
    const int whole = a.k / kScaleBlock;
    for (int b = wave; b < whole; b += waves) block(b, std::false_type{});
    if (whole < a.k_blocks && whole % waves == wave) block(whole, std::true_type{});
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
    }
}

template <int MT, int NT, bool EXACT, bool GROUPED>
void launch_direct(const ProductArgs &a, int64_t row_tiles, int waves, hipStream_t s) {
  const dim3 grid((unsigned)((a.n + 16 * NT - 1) / (16 * NT)), (unsigned)row_tiles);
  hipLaunchKernelGGL((lutkan_fp8_direct_kernel<MT, NT, EXACT, GROUPED>), grid, dim3(64 * waves), waves > 1 ? (size_t)waves * MT * NT * 64 * sizeof(f32x4) : 0, s, a);
}

// A tile of 16 MT WM rows x 16 NT WN columns for a work-group of WM x WN waves, each 16 MT rows x 16 NT columns of it.  Both operands'
// blocks of k go through LDS, in two buffers of 128 bytes a row: while a block is multiplied the next is on its way.  A row's eight
// 16-byte pieces lie in an order that depends on the row (piece_place), so that the 16 rows that a read of 16 lanes takes lie in
// different banks.
//   ASYNC: the pieces go from global memory to LDS without passing through registers: needs 16-byte aligned rows and offsets
//   that fit 32 bits.  Otherwise, and for a last block that is not whole, through registers.
__device__ __forceinline__ int piece_place(int row, int piece) { return piece ^ ((row >> 1) & 7); }

template <int MT, int NT, int WM, int WN, bool EXACT, bool GROUPED, bool ASYNC>
__global__ __launch_bounds__(64 * WM * WN, 512 / (64 * WM * WN)) void lutkan_fp8_tiled_kernel(const ProductArgs a, unsigned row_tiles) {
  constexpr int kRows = 16 * MT * WM, kCols = 16 * NT * WN, kWaves = WM * WN, kThreads = 64 * kWaves, kStage = (kRows + kCols) * kScaleBlock;
  constexpr int kXCopies = kRows / 8 / kWaves, kWCopies = kCols / 8 / kWaves;          // of 8 rows, for each wave
  static_assert(kXCopies * 8 * kWaves == kRows && kWCopies * 8 * kWaves == kCols && kThreads >= kRows && kScaleBlock % (16 * NT) == 0, "tile");
  extern __shared__ __align__(16) unsigned char s_tiles[];       // [buffer][rows of x, rows of the weight][128], then [buffer][threads] scales
  float *s_scales = reinterpret_cast<float *>(s_tiles + 2 * kStage);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave / WN, wn = wave % WN, p = lane >> 4;
  // Work-groups go to the eight XCDs in turn: each XCD gets a run of neighbouring tiles, and in a run eight row tiles share a column
  // tile before the next, so that what an XCD's work-groups read at a time meets in its L2.
  const unsigned col_tiles = (a.n + kCols - 1) / kCols;
  if constexpr (GROUPED) row_tiles = (unsigned)uniform(grouped_tiles(a, kRows));
  const unsigned tiles = row_tiles * col_tiles;
  if (blockIdx.x >= tiles) return;
  const unsigned xcd = blockIdx.x % 8, of_xcd = tiles / 8, more = tiles % 8;
  const unsigned tile = xcd * of_xcd + min(xcd, more) + blockIdx.x / 8;
  const unsigned band = tile / (8 * col_tiles), in_band = tile - band * 8 * col_tiles, high = min(8u, row_tiles - band * 8);
  const unsigned row_tile = band * 8 + in_band % high;
  const int col0 = (int)(in_band / high) * kCols;
  RowTile t;
  if constexpr (GROUPED) {
    t = grouped_tile(a, row_tile, kRows);
    t.first = uniform(t.first); t.end = uniform(t.end); t.group = __builtin_amdgcn_readfirstlane(t.group);
  } else {
    t.first = (int64_t)row_tile * kRows;
    t.end = min(t.first + kRows, a.rows);
    t.group = 0;
  }
  f32x4 acc[MT][NT];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[m][n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  if (t.group >= 0) {
    const unsigned char *w_tile = a.w + t.group * a.w_matrix_stride + (int64_t)col0 * a.w_stride;
    const unsigned char *x_tile = GROUPED ? a.x : a.x + t.first * a.x_stride;
    typedef std::conditional_t<ASYNC, unsigned, int64_t> offset_t;
    offset_t x_from[kXCopies], w_from[kWCopies];                 // the rows that this lane's pieces come from
    int piece_at[2];                                             // and the columns: place i of row r, the same for every 16 rows
#pragma unroll
    for (int c = 0; c < 2; ++c) piece_at[c] = piece_place(c * 8 + (lane >> 3), lane & 7) * 16;        // (its own inverse)
    static_assert(kXCopies % 2 == 0 && kWCopies % 2 == 0, "copies in pairs");
#pragma unroll
    for (int c = 0; c < kXCopies; ++c) {
      const int64_t row = min(t.first + (wave * kXCopies + c) * 8 + (lane >> 3), t.end - 1);
      x_from[c] = (offset_t)((GROUPED ? max(source_row<GROUPED>(a, row), (int64_t)0) : row - t.first) * a.x_stride);
    }
#pragma unroll
    for (int c = 0; c < kWCopies; ++c) w_from[c] = (offset_t)((int64_t)min((wave * kWCopies + c) * 8 + (lane >> 3), a.n - 1 - col0) * a.w_stride);
    const int64_t scale_row = min(t.first + min(tid, kRows - 1), t.end - 1);
    const float *xs = a.x_scales + max(source_row<GROUPED>(a, scale_row), (int64_t)0) * a.x_scales_stride;
    const float *ws = a.w_scales + ((int64_t)t.group * a.n_blocks + min(col0 + wn * 16 * NT, a.n - 1) / kScaleBlock) * a.k_blocks;
    const int whole = a.k / kScaleBlock;
    u32x4 held[ASYNC ? 1 : kXCopies + kWCopies];
    // Block b's pieces are asked for, and put into a buffer: at once where they go straight there, else by put().
    const auto ask = [&](int b) {
      if constexpr (ASYNC) {
        unsigned char *to = s_tiles + (b & 1) * kStage;
#pragma unroll
        for (int c = 0; c < kXCopies; ++c) copy16_global_to_lds_at(x_tile + (int64_t)b * kScaleBlock, x_from[c] + piece_at[c & 1], to + (wave * kXCopies + c) * 1024);
#pragma unroll
        for (int c = 0; c < kWCopies; ++c)
          copy16_global_to_lds_at(w_tile + (int64_t)b * kScaleBlock, w_from[c] + piece_at[c & 1], to + kRows * kScaleBlock + (wave * kWCopies + c) * 1024);
      } else {
#pragma unroll
        for (int c = 0; c < kXCopies; ++c) held[c] = load_any<u32x4>(x_tile + x_from[c] + (b * kScaleBlock + piece_at[c & 1]));
#pragma unroll
        for (int c = 0; c < kWCopies; ++c) held[kXCopies + c] = load_any<u32x4>(w_tile + w_from[c] + (b * kScaleBlock + piece_at[c & 1]));
      }
    };
    const auto put = [&](int b) {
      if constexpr (!ASYNC) {
        unsigned char *to = s_tiles + (b & 1) * kStage + lane * 16;
#pragma unroll
        for (int c = 0; c < kXCopies; ++c) *reinterpret_cast<u32x4 *>(to + (wave * kXCopies + c) * 1024) = held[c];
#pragma unroll
        for (int c = 0; c < kWCopies; ++c) *reinterpret_cast<u32x4 *>(to + kRows * kScaleBlock + (wave * kWCopies + c) * 1024) = held[kXCopies + c];
      }
    };
    // The last block, if it is not whole.
    const auto put_end = [&]() {
      unsigned char *to = s_tiles + (whole & 1) * kStage + lane * 16;
      for (int c = 0; c < kXCopies; ++c)
        *reinterpret_cast<u32x4 *>(to + (wave * kXCopies + c) * 1024) = piece_at_end(x_tile + x_from[c], whole * kScaleBlock + piece_at[c & 1], a.k);
      for (int c = 0; c < kWCopies; ++c)
        *reinterpret_cast<u32x4 *>(to + kRows * kScaleBlock + (wave * kWCopies + c) * 1024) = piece_at_end(w_tile + w_from[c], whole * kScaleBlock + piece_at[c & 1], a.k);
    };
    const int at_row = lane & 15, low = at_row * kScaleBlock + piece_place(at_row, p) * 16, high_half = at_row * kScaleBlock + piece_place(at_row, p + 4) * 16;
    // One block: the products in a fixed order, each added two products after it was begun; a row subtile's codes are read while the one
    // before it is multiplied.
    const auto multiply = [&](int b, float w_scale) {
      const unsigned char *xt = s_tiles + (b & 1) * kStage + (wm * 16 * MT) * kScaleBlock;
      const unsigned char *wt = s_tiles + (b & 1) * kStage + (kRows + wn * 16 * NT) * kScaleBlock;
      const float *scales = s_scales + (b & 1) * kThreads + wm * 16 * MT + at_row;
      const auto codes = [&](const unsigned char *rows, int sub) {
        return fragment(*reinterpret_cast<const u32x4 *>(rows + sub * 16 * kScaleBlock + low), *reinterpret_cast<const u32x4 *>(rows + sub * 16 * kScaleBlock + high_half));
      };
      Operand<EXACT> wf[NT];
#pragma unroll
      for (int n = 0; n < NT; ++n) wf[n].set(codes(wt, n));
      i32x8 next = codes(xt, 0);
      float next_scale = scales[0];
      Operand<EXACT> xf;
      f32x4 v[3];
      float scales_of[2];
#pragma unroll
      for (int i = 0; i < MT * NT + 2; ++i) {
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
          v[i % 3] = block_product(wf[n], xf);
        }
        if (i >= 2) {
          const int of = i - 2;
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[of / NT][of % NT][e] = fmaf(scales_of[(of / NT) & 1], v[of % 3][e], acc[of / NT][of % NT][e]);
          asm volatile("" : "+v"(acc[of / NT][of % NT]));        // (here, not behind the next branch, with all products held until then)
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    float scale = xs[0], w_scale = ws[0];
    if (whole > 0) {
      ask(0);
      put(0);
    }
    s_scales[tid] = scale;                                       // (threads beyond the rows: the last row's again, behind the others)
    for (int b = 0; b < whole; ++b) {
      wait_all_vector_loads();
      lds_barrier();                                             // block b is there, and nobody reads the other buffer any more
      scale = xs[min(b + 1, a.k_blocks - 1)];                    // (before the copies: a wait for these does not have to wait for them)
      const float next_w_scale = ws[min(b + 1, a.k_blocks - 1)];
      if (b + 1 < whole) ask(b + 1);
      multiply(b, w_scale);
      w_scale = next_w_scale;
      if (b + 1 < whole) put(b + 1);
      s_scales[((b + 1) & 1) * kThreads + tid] = scale;
    }
    if (whole < a.k_blocks) {
      put_end();                                                 // (into the buffer that nobody reads since the last barrier)
      lds_barrier();
      multiply(whole, w_scale);
    }
  }
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    const int64_t row = t.first + (wm * MT + m) * 16 + (lane & 15);
    if (row >= t.end) continue;
    const bool none = t.group < 0 || source_row<GROUPED>(a, row) < 0;
#pragma unroll
    for (int n = 0; n < NT; ++n) store_outputs(a, row, col0 + (wn * NT + n) * 16 + 4 * p, none ? f32x4{0.0f, 0.0f, 0.0f, 0.0f} : acc[m][n]);
  }
}

template <int MT, int NT, int WM, int WN, bool EXACT, bool GROUPED, bool ASYNC>
int launch_tiled(const ProductArgs &a, int64_t row_tiles, const char *who, hipStream_t s) {
  constexpr int kRows = 16 * MT * WM, kCols = 16 * NT * WN;
  constexpr int kLds = 2 * (kRows + kCols) * kScaleBlock + 2 * 64 * WM * WN * (int)sizeof(float);
  static LdsCap cap;
  const auto kernel = lutkan_fp8_tiled_kernel<MT, NT, WM, WN, EXACT, GROUPED, ASYNC>;
  if (int rc = raise_lds_cap(kernel, &cap, who)) return rc;
  lutkan::plan_note("fp8_tiled rows=%d columns=%d%s; ", kRows, kCols, ASYNC ? " async" : "");
  hipLaunchKernelGGL(kernel, dim3((unsigned)(row_tiles * ((a.n + kCols - 1) / kCols))), dim3(64 * WM * WN), kLds, s, a, (unsigned)row_tiles);
  return check_launch(who);
}

template <int MT, int NT, int WM, int WN, bool EXACT, bool GROUPED>
int launch_tiled(const ProductArgs &a, int64_t row_tiles, const char *who, hipStream_t s) {
  const int64_t x_span = (GROUPED ? a.x_rows : 16 * MT * WM) * a.x_stride, w_span = 16 * NT * WN * a.w_stride;
  const bool async = ((reinterpret_cast<uintptr_t>(a.x) | reinterpret_cast<uintptr_t>(a.w) | (uintptr_t)a.x_stride | (uintptr_t)a.w_stride | (uintptr_t)a.w_matrix_stride) & 15) == 0 &&
                     x_span < ((int64_t)1 << 32) && w_span < ((int64_t)1 << 32);
  return async ? launch_tiled<MT, NT, WM, WN, EXACT, GROUPED, true>(a, row_tiles, who, s) : launch_tiled<MT, NT, WM, WN, EXACT, GROUPED, false>(a, row_tiles, who, s);
}

template <bool EXACT, bool GROUPED>
int launch_product(const ProductArgs &a, const char *who, hipStream_t s) {
  const int groups = GROUPED ? a.groups : 1;
  const auto tiles = [&](int height) {                           // no routing has more
    return GROUPED ? a.rows / height + std::min<int64_t>(groups + 1, a.rows) : (a.rows + height - 1) / height;
  };
  if (tiles(64) * ((a.n + 63) / 64) > 0x7fffffff) return fail(LUTKAN_EUNSUPPORTED, "%s: too many outputs", who);
  lutkan::plan_clear();
  const int64_t large = tiles(256) * ((a.n + 255) / 256);        // (at least three quarters of the compute units get a tile)
  int pick = a.rows <= 32 * (int64_t)groups ? 0 : a.rows < 128 * (int64_t)groups ? 1 : EXACT || large < 192 ? 2 : 3;
  if (pick == 0) {
    if (tiles(16) > 65535) return fail(LUTKAN_EUNSUPPORTED, "%s: too many rows", who);
    const int waves = std::max(1, std::min(a.k_blocks, 16));
    lutkan::plan_note("fp8_direct rows=16 columns=16 waves=%d; ", waves);
    launch_direct<1, 1, EXACT, GROUPED>(a, tiles(16), waves, s);
  } else if (pick == 1) {
    if (tiles(64) > 65535) return fail(LUTKAN_EUNSUPPORTED, "%s: too many rows", who);
    const int waves = std::max(1, std::min(a.k_blocks, 4));
    lutkan::plan_note("fp8_direct rows=64 columns=64 waves=%d; ", waves);
    launch_direct<4, 4, EXACT, GROUPED>(a, tiles(64), waves, s);
  } else {
    if constexpr (EXACT) return launch_tiled<4, 4, 2, 2, EXACT, GROUPED>(a, tiles(128), who, s);
    else return pick == 2 ? launch_tiled<4, 4, 2, 2, EXACT, GROUPED>(a, tiles(128), who, s) : launch_tiled<8, 4, 2, 4, EXACT, GROUPED>(a, tiles(256), who, s);
  }
  return check_launch(who);
}

int check_product(const lutkan_matmul_fp8_args *p, const char *who, ProductArgs *a) {
  if (!p) return fail(LUTKAN_EINVAL, "%s: null arguments", who);
  if (p->rows < 0 || p->x_rows < 0 || p->k < 1 || p->n < 1) return fail(LUTKAN_EINVAL, "%s: rows %lld of %lld, %d x %d", who, (long long)p->rows, (long long)p->x_rows, p->n, p->k);
  if (p->k > LUTKAN_FP8_MAX_INPUTS) return fail(LUTKAN_EUNSUPPORTED, "%s: %d inputs, at most %d", who, p->k, LUTKAN_FP8_MAX_INPUTS);
  if (p->n > LUTKAN_FP8_MAX_INPUTS) return fail(LUTKAN_EUNSUPPORTED, "%s: %d outputs, at most %d", who, p->n, LUTKAN_FP8_MAX_INPUTS);
  if (!is_type(p->y_type)) return fail(LUTKAN_EINVAL, "%s: bad type", who);
  if (p->rows > 0 && (!p->x || !p->x_scales || !p->weight || !p->weight_scales || !p->y)) return fail(LUTKAN_EINVAL, "%s: null x / x_scales / weight / weight_scales / y", who);
  const int64_t k_blocks = scale_blocks(p->k);
  if (p->y_stride < p->n) return fail(LUTKAN_ESHAPE, "%s: a row of y is longer than its stride", who);
  if (p->x_stride < 0 || p->weight_stride < 0 || p->x_scales_stride < 0 || p->weight_matrix_stride < 0) return fail(LUTKAN_ESHAPE, "%s: negative stride", who);
  *a = ProductArgs{};
  a->x = static_cast<const unsigned char *>(p->x); a->w = static_cast<const unsigned char *>(p->weight);
  a->x_scales = p->x_scales; a->w_scales = p->weight_scales; a->y = static_cast<unsigned char *>(p->y);
  a->x_rows = p->x_rows; a->x_stride = p->x_stride; a->x_scales_stride = p->x_scales_stride;
  a->w_stride = p->weight_stride; a->w_matrix_stride = p->weight_matrix_stride; a->y_stride = p->y_stride;
  a->rows = p->rows; a->k = p->k; a->n = p->n; a->k_blocks = (int32_t)k_blocks; a->n_blocks = (int32_t)scale_blocks(p->n); a->y_type = p->y_type;
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
  if (p->rows == 0) return LUTKAN_OK;
  if (!p->group_sizes) return fail(LUTKAN_EINVAL, "%s: null group_sizes", who);
  if ((p->group_sizes_bytes != 4 && p->group_sizes_bytes != 8) || (p->row_index && p->row_index_bytes != 4 && p->row_index_bytes != 8))
    return fail(LUTKAN_EINVAL, "%s: group_sizes and row_index are whole numbers of 4 or 8 bytes", who);
  if (!p->row_index && p->rows != p->x_rows) return fail(LUTKAN_ESHAPE, "%s: %lld rows out, %lld in, and no row_index", who, (long long)p->rows, (long long)p->x_rows);
  if (p->row_index && p->x_rows == 0) return fail(LUTKAN_ESHAPE, "%s: row_index into no rows", who);
  a.group_sizes = p->group_sizes; a.row_index = p->row_index; a.groups = p->groups;
  a.group_sizes_bytes = p->group_sizes_bytes; a.row_index_bytes = p->row_index_bytes;
  return a.y_type == LUTKAN_F32 ? launch_product<true, true>(a, who, s) : launch_product<false, true>(a, who, s);
}
