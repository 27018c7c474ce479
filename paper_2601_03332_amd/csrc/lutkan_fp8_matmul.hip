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
// itself, a lane a group, 64 groups at a time.
__device__ __forceinline__ RowTile grouped_tile(const ProductArgs &a, int64_t tile, int height) {
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
  const int64_t at = row0 + (tile - tile0) * height;
  return {at, min(at + height, a.rows), -1};
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

template <bool EXACT, bool GROUPED>
int launch_product(const ProductArgs &a, const char *who, hipStream_t s) {
  const int groups = GROUPED ? a.groups : 1;
  const auto tiles = [&](int height) {                           // no routing has more
    return GROUPED ? a.rows / height + std::min<int64_t>(groups + 1, a.rows) : (a.rows + height - 1) / height;
  };
  const bool few = a.rows <= 32 * (int64_t)groups;
  const int height = few ? 16 : 64;
  if (tiles(height) > 65535) return fail(LUTKAN_EUNSUPPORTED, "%s: too many rows", who);
  lutkan::plan_clear();
  if (few) {
    const int waves = std::max(1, std::min(a.k_blocks, 16));
    lutkan::plan_note("fp8_direct rows=16 columns=16 waves=%d; ", waves);
    launch_direct<1, 1, EXACT, GROUPED>(a, tiles(16), waves, s);
  } else {
    const int waves = std::max(1, std::min(a.k_blocks, 4));
    lutkan::plan_note("fp8_direct rows=64 columns=64 waves=%d; ", waves);
    launch_direct<4, 4, EXACT, GROUPED>(a, tiles(64), waves, s);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(LUTKAN_EHIP, "%s: %s", who, hipGetErrorString(e));
  return LUTKAN_OK;
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
