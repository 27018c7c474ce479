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

// Scales that fp32 multiplies without loss: a product of two lies in 2^-120 .. 2^120, and times a sum below 2^31 beyond fp32 only where y is.
__device__ __forceinline__ bool ordinary(float scale) { return scale >= 0x1p-60f && scale <= 0x1p60f; }

// Four sums times their scales; `exact`: in fp64, for scales that are not ordinary (uniform over a wave).
__device__ __forceinline__ f32x4 scaled(i32x4 sum, float x_scale, f32x4 w_scale, bool exact) {
  f32x4 v;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    v[e] = exact ? (float)((double)sum[e] * ((double)x_scale * (double)w_scale[e])) : (float)sum[e] * (x_scale * w_scale[e]);
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
      const float xs = from[m] >= 0 ? a.x_scales[from[m] * a.x_scales_stride] : 1.0f;
      const f32x4 ws = weight_scales(a, max(t.group, 0), col);
      const bool exact = !__all(ordinary(xs) && ordinary(ws[0]) && ordinary(ws[1]) && ordinary(ws[2]) && ordinary(ws[3]));
      if (from[m] >= 0) y = scaled(v, xs, ws, exact);
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

template <bool GROUPED>
int launch_product(const ProductArgs &a, const char *who, hipStream_t s) {
  const int64_t groups = GROUPED ? a.groups : 1;
  const auto tiles = [&](int height) {                           // no routing has more
    return GROUPED ? a.rows / height + std::min<int64_t>(groups + 1, a.rows) : ((int64_t)a.rows + height - 1) / height;
  };
  lutkan::plan_clear();
  return launch_direct<2, 2, GROUPED>(a, tiles(32), rows_aligned(a), who, s);
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
