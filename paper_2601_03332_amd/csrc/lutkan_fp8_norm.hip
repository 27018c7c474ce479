// Conversion to 8-bit floating point (e4m3) with a scale for each 128 columns of a row, after the residual's addition and the
// root-mean-square norm, and of a weight with a scale for each block of 128 x 128.
#include "lutkan_fp8.h"

namespace {

// (A launch whose arguments take at most 112 bytes costs the host 2.8 us, one with 160 bytes 3.5: strides travel in 32 bits.)
struct NormArgs {
  const unsigned char *x, *residual, *weight;
  unsigned char *residual_out, *codes;
  float *scales;
  int64_t rows;
  int32_t x_stride, residual_stride, residual_out_stride, codes_stride, scales_stride;   // elements from one row to the next
  int32_t width, weight_type, row_waves;
  float eps, inverse_width;
};
static_assert(sizeof(NormArgs) <= 112, "launch");

constexpr int kNoResidual = -1, kRowsOfGroup = 4;

// One row is normalised by `row_waves` waves, 64 * 8 * CH columns each; a work-group holds one row, or (row_waves = 1) four.  Every
// element is read once, stays in a register as fp32, and leaves as its sum with the residual and as its code: lane l of a row's
// lanes holds the eight columns 8 (l + lanes c), c < CH, so that 16 neighbouring lanes hold one block of 128.
// Bound by memory: 32768 rows of 1024 (bf16, residual bf16) 47 us, 5.0 TB/s, where a copy of 1 GiB reaches 5.1; with several waves a row
// 8192 rows of 4096 42 - 47 us (5.6 - 5.0), 4096 of 8192 44, 2048 of 16384 46, 1024 of 32768 56 (4.3; a work-group of 16 waves has the compute unit to
// itself).  A few rows: the host, 5.9 us a call for one row of 1024; its kernel is 2.8, one dependent chain of load, two reductions and store.
template <int X, int R, int CH>
__global__ __launch_bounds__(1024) void lutkan_rmsnorm_fp8_kernel(const NormArgs a) {
  const int row_waves = a.row_waves;
  __shared__ float s_sum[16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t row = row_waves == 1 ? (int64_t)blockIdx.x * kRowsOfGroup + wave : blockIdx.x;
  if (row >= a.rows) return;                                     // (whole waves of a work-group without a barrier)
  const int lanes = row_waves * 64, at = row_waves == 1 ? lane : threadIdx.x;
  const unsigned char *x = a.x + row * a.x_stride * type_bytes(X);
  float h[CH][8];
  {
    Raw8<X> rx[CH];
    Raw8<R == kNoResidual ? LUTKAN_BF16 : R> rr[CH];
    const unsigned char *r = R == kNoResidual ? nullptr : a.residual + row * a.residual_stride * type_bytes(R);
#pragma unroll
    for (int c = 0; c < CH; ++c) {                               // all loads of the row first
      const int col = 8 * (at + lanes * c);
      if (col + 8 <= a.width) {
        rx[c] = load_raw8<X>(x + (size_t)col * type_bytes(X));
        if constexpr (R != kNoResidual) rr[c] = load_raw8<R>(r + (size_t)col * type_bytes(R));
      }
    }
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int col = 8 * (at + lanes * c);
      if (col + 8 <= a.width) {
        values8<X>(rx[c], h[c]);
        if constexpr (R != kNoResidual) {
          float v[8];
          values8<R>(rr[c], v);
#pragma unroll
          for (int e = 0; e < 8; ++e) h[c][e] += v[e];
        }
      } else {                                                   // the row ends inside these eight columns, or before them
#pragma unroll
        for (int e = 0; e < 8; ++e) h[c][e] = 0.0f;
        if (col >= a.width) continue;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if (col + e < a.width) {
            h[c][e] = load_one<X>(x + (size_t)(col + e) * type_bytes(X));
            if constexpr (R != kNoResidual) h[c][e] += load_one<R>(r + (size_t)(col + e) * type_bytes(R));
          }
        }
      }
    }
  }
  const auto read_weight = [&](int col, float (&weight)[8]) {
    if (col + 8 <= a.width) {
      if (a.weight_type == LUTKAN_F32) values8<LUTKAN_F32>(load_raw8<LUTKAN_F32>(a.weight + (size_t)col * 4), weight);
      else if (a.weight_type == LUTKAN_F16) values8<LUTKAN_F16>(load_raw8<LUTKAN_F16>(a.weight + (size_t)col * 2), weight);
      else values8<LUTKAN_BF16>(load_raw8<LUTKAN_BF16>(a.weight + (size_t)col * 2), weight);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) weight[e] = 0.0f;
      if (col < a.width) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if (col + e >= a.width) continue;
          const unsigned char *w = a.weight + (size_t)(col + e) * type_bytes(a.weight_type);
          weight[e] = a.weight_type == LUTKAN_F32 ? load_one<LUTKAN_F32>(w) : a.weight_type == LUTKAN_F16 ? load_one<LUTKAN_F16>(w) : load_one<LUTKAN_BF16>(w);
        }
      }
    }
  };
  float first_weight[8];                                         // of a lane's only columns: asked for before the sum is known
  if constexpr (CH == 1) read_weight(8 * at, first_weight);      // (with more of them it costs registers: 32768 rows of 1024 47 -> 50 us)
  const auto sum_of_squares = [&](float factor) {
    float sum = 0.0f;
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) sum = fmaf(h[c][e] * factor, h[c][e] * factor, sum);
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off);
    if (row_waves > 1) {
      if (lane == 0) s_sum[wave] = sum;
      __syncthreads();
      sum = 0.0f;
      for (int w = 0; w < row_waves; ++w) sum += s_sum[w];
    }
    return sum;
  };
  const float sum = sum_of_squares(1.0f), mean = fmaf(sum, a.inverse_width, a.eps);
  float factor = 1.0f, inverse_rms = 1.0f / sqrtf(mean);
  // Squares beyond fp32 (|h| above 1.8e19, or a row that holds an infinity or NaN) or below what it holds well: both over again with h times a power of 2.
  // The largest |h| squared is then 2^96, the smallest that can bring a row here 2^-24; a sum that is too small was below 2^-85, now 2^115.
  if (!(finite(sum) && mean >= 0x1p-100f)) {
    factor = finite(sum) ? 0x1p100f : 0x1p-80f;
    if (row_waves > 1) __syncthreads();                          // (the row is the work-group's: all its waves are here, and have read the first sum)
    inverse_rms = 1.0f / sqrtf(fmaf(sum_of_squares(factor), a.inverse_width, a.eps * factor * factor));
  }
  unsigned char *codes = a.codes + row * a.codes_stride;
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const int col = 8 * (at + lanes * c);
    const bool whole = col + 8 <= a.width;
    float y[8], weight[8];
    if constexpr (CH > 1) read_weight(col, weight);
    unsigned largest = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      y[e] = h[c][e] * factor * inverse_rms * (CH == 1 ? first_weight[e] : weight[e]);
      if (whole || col + e < a.width) largest = max(largest, magnitude(y[e]));      // (0 * an infinite norm beyond the row's end is none of its values)
    }
#pragma unroll
    for (int off = 8; off > 0; off >>= 1) largest = max(largest, (unsigned)__shfl_xor((int)largest, off));
    const float scale = block_scale(largest);
    const u32x2 code = codes8(y, scale);
    if ((at & 15) == 0 && col < a.width) a.scales[row * a.scales_stride + col / kScaleBlock] = scale;
    if (whole) {
      store_any(codes + col, code);
      if constexpr (R != kNoResidual) store8<R>(a.residual_out + (row * a.residual_out_stride + col) * type_bytes(R), h[c]);
    } else if (col < a.width) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (col + e < a.width) {
          codes[col + e] = (unsigned char)(code[e >> 2] >> ((e & 3) * 8));
          if constexpr (R != kNoResidual) store_one<R>(a.residual_out + (row * a.residual_out_stride + col + e) * type_bytes(R), h[c][e]);
        }
    }
  }
}

template <int X, int R>
void launch_norm(const NormArgs &a, int chunks, unsigned groups, unsigned threads, hipStream_t s) {
  switch (chunks) {
    case 1: hipLaunchKernelGGL((lutkan_rmsnorm_fp8_kernel<X, R, 1>), dim3(groups), dim3(threads), 0, s, a); break;
    case 2: hipLaunchKernelGGL((lutkan_rmsnorm_fp8_kernel<X, R, 2>), dim3(groups), dim3(threads), 0, s, a); break;
    default: hipLaunchKernelGGL((lutkan_rmsnorm_fp8_kernel<X, R, 4>), dim3(groups), dim3(threads), 0, s, a); break;
  }
}

template <int X>
void launch_norm_of(const NormArgs &a, int residual_type, int chunks, unsigned groups, unsigned threads, hipStream_t s) {
  switch (a.residual ? residual_type : kNoResidual) {
    case LUTKAN_F32: launch_norm<X, LUTKAN_F32>(a, chunks, groups, threads, s); break;
    case LUTKAN_F16: launch_norm<X, LUTKAN_F16>(a, chunks, groups, threads, s); break;
    case LUTKAN_BF16: launch_norm<X, LUTKAN_BF16>(a, chunks, groups, threads, s); break;
    default: launch_norm<X, kNoResidual>(a, chunks, groups, threads, s); break;
  }
}

struct QuantiseArgs {
  const unsigned char *w;
  unsigned char *codes;
  float *scales;
  int64_t w_stride, w_matrix_stride;
  int32_t n, k;
  unsigned first;                                                // block of the launch's first work-group
};

// A work-group of 256 threads converts one block: 16 lanes a row of 128 columns, eight rows each thread, all in registers between
// the one read and the one write.
// Bound by memory: 4096 x 4096 bf16 9.6 us, 5.2 TB/s.
template <int X>
__global__ __launch_bounds__(256) void lutkan_quantise_fp8_kernel(const QuantiseArgs a) {
  __shared__ unsigned s_largest[4];
  const unsigned column_blocks = ((unsigned)a.k + kScaleBlock - 1) / kScaleBlock, row_blocks = ((unsigned)a.n + kScaleBlock - 1) / kScaleBlock;
  const unsigned block = a.first + blockIdx.x, column_block = block % column_blocks, rest = block / column_blocks, row_block = rest % row_blocks;
  const int64_t matrix = rest / row_blocks;
  const int col = column_block * kScaleBlock + 8 * (threadIdx.x & 15), row0 = row_block * kScaleBlock + (threadIdx.x >> 4);
  const unsigned char *w = a.w + (matrix * a.w_matrix_stride + col) * type_bytes(X);
  const bool whole = a.k - col >= 8;                             // (col + 8 can pass 2^31)
  float v[8][8];
  if (whole) {                                                   // all loads first; rows behind the last are the last again
    Raw8<X> raw[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) raw[i] = load_raw8<X>(w + min(row0 + 16 * i, a.n - 1) * a.w_stride * type_bytes(X));
#pragma unroll
    for (int i = 0; i < 8; ++i) values8<X>(raw[i], v[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] = 0.0f;
    if (col < a.k)                                               // the rows end inside these eight columns
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (col + e < a.k)
#pragma unroll
          for (int i = 0; i < 8; ++i) v[i][e] = load_one<X>(w + (min(row0 + 16 * i, a.n - 1) * a.w_stride + e) * type_bytes(X));
  }
  unsigned largest = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) largest = max(largest, magnitude(v[i][e]));
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) largest = max(largest, (unsigned)__shfl_xor((int)largest, off));
  if ((threadIdx.x & 63) == 0) s_largest[threadIdx.x >> 6] = largest;
  __syncthreads();
  largest = max(max(s_largest[0], s_largest[1]), max(s_largest[2], s_largest[3]));
  const float scale = block_scale(largest);
  if (threadIdx.x == 0) a.scales[block] = scale;                // the blocks' order is the scales'
  unsigned char *codes = a.codes + matrix * a.n * a.k + col;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int row = row0 + 16 * i;
    if (row >= a.n) continue;
    const u32x2 code = codes8(v[i], scale);
    if (whole) {
      store_any(codes + (int64_t)row * a.k, code);
    } else if (col < a.k) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (col + e < a.k) codes[(int64_t)row * a.k + e] = (unsigned char)(code[e >> 2] >> ((e & 3) * 8));
    }
  }
}

}  // namespace

extern "C" int lutkan_rmsnorm_fp8(const lutkan_rmsnorm_fp8_args *p, void *hip_stream) {
  const char *who = "lutkan_rmsnorm_fp8";
  if (!p) return fail(LUTKAN_EINVAL, "%s: null arguments", who);
  if (p->rows < 0 || p->width < 1) return fail(LUTKAN_EINVAL, "%s: rows %lld, width %d", who, (long long)p->rows, p->width);
  if (p->width > LUTKAN_FP8_MAX_WIDTH) return fail(LUTKAN_EUNSUPPORTED, "%s: width %d, at most %d", who, p->width, LUTKAN_FP8_MAX_WIDTH);
  if (!is_type(p->x_type) || !is_type(p->weight_type) || (p->residual && !is_type(p->residual_type))) return fail(LUTKAN_EINVAL, "%s: bad type", who);
  if (!(p->eps >= 0.0f)) return fail(LUTKAN_EINVAL, "%s: eps must be >= 0", who);
  if (p->rows == 0) return LUTKAN_OK;
  if (!p->x || !p->weight || !p->codes || !p->scales) return fail(LUTKAN_EINVAL, "%s: null x / weight / codes / scales", who);
  if ((p->residual != nullptr) != (p->residual_out != nullptr)) return fail(LUTKAN_EINVAL, "%s: residual and residual_out come together", who);
  const int64_t blocks = scale_blocks(p->width);
  if (p->codes_stride < p->width || p->scales_stride < blocks || (p->residual && p->residual_out_stride < p->width))
    return fail(LUTKAN_ESHAPE, "%s: a row of the outputs is longer than its stride", who);
  if (p->x_stride < 0 || (p->residual && p->residual_stride < 0)) return fail(LUTKAN_ESHAPE, "%s: negative stride", who);
  if (std::max({p->x_stride, p->codes_stride, p->scales_stride, p->residual ? p->residual_stride : 0, p->residual ? p->residual_out_stride : 0}) > INT32_MAX)
    return fail(LUTKAN_EUNSUPPORTED, "%s: row strides of at most 2^31 - 1", who);
  // Waves to a row: one while the launch fills the GPU with a wave a row and the row fits its registers; else enough for eight
  // columns a lane, so that a few rows are spread over many lanes.
  int waves = (p->width + 511) / 512, chunks = 1;
  if (p->rows >= 2048 && waves <= 4) { chunks = waves; waves = 1; }
  else if (p->rows >= 1024 && waves <= 16) { chunks = waves > 8 ? 4 : waves > 4 ? 2 : 1; waves = (waves + chunks - 1) / chunks; }
  while (waves > 16) { chunks *= 2; waves = (p->width + 512 * chunks - 1) / (512 * chunks); }
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const unsigned threads = waves == 1 ? 64u * kRowsOfGroup : (unsigned)waves * 64u;
  const int group_rows = waves == 1 ? kRowsOfGroup : 1;
  const int64_t launch_rows = lutkan::kMaxLaunchThreads / threads * group_rows;          // (more rows: more launches)
  const int64_t residual_bytes = p->residual ? type_bytes(p->residual_type) : 0;
  for (int64_t first = 0; first < p->rows; first += launch_rows) {
    NormArgs a;
    a.x = static_cast<const unsigned char *>(p->x) + first * p->x_stride * type_bytes(p->x_type);
    a.residual = static_cast<const unsigned char *>(p->residual) + first * p->residual_stride * residual_bytes;
    a.weight = static_cast<const unsigned char *>(p->weight);
    a.residual_out = static_cast<unsigned char *>(p->residual_out) + first * p->residual_out_stride * residual_bytes;
    a.codes = static_cast<unsigned char *>(p->codes) + first * p->codes_stride; a.scales = p->scales + first * p->scales_stride;
    a.x_stride = (int32_t)p->x_stride; a.residual_stride = (int32_t)p->residual_stride; a.residual_out_stride = (int32_t)p->residual_out_stride;
    a.codes_stride = (int32_t)p->codes_stride; a.scales_stride = (int32_t)p->scales_stride; a.row_waves = waves;
    a.rows = std::min(p->rows - first, launch_rows); a.width = p->width; a.weight_type = p->weight_type;
    a.eps = p->eps; a.inverse_width = 1.0f / (float)p->width;
    const unsigned groups = (unsigned)((a.rows + group_rows - 1) / group_rows);
    switch (p->x_type) {
      case LUTKAN_F32: launch_norm_of<LUTKAN_F32>(a, p->residual_type, chunks, groups, threads, s); break;
      case LUTKAN_F16: launch_norm_of<LUTKAN_F16>(a, p->residual_type, chunks, groups, threads, s); break;
      default: launch_norm_of<LUTKAN_BF16>(a, p->residual_type, chunks, groups, threads, s); break;
    }
    if (int rc = check_launch(who)) return rc;
  }
  return LUTKAN_OK;
}

extern "C" int lutkan_quantise_fp8(const void *weight, int32_t type, int64_t matrices, int32_t n, int32_t k, int64_t stride, int64_t matrix_stride,
                                   void *codes, float *scales, void *hip_stream) {
  const char *who = "lutkan_quantise_fp8";
  if (!is_type(type)) return fail(LUTKAN_EINVAL, "%s: bad type", who);
  if (matrices < 0 || n < 1 || k < 1) return fail(LUTKAN_EINVAL, "%s: %lld matrices of %d x %d", who, (long long)matrices, n, k);
  if (matrices == 0) return LUTKAN_OK;
  if (!weight || !codes || !scales) return fail(LUTKAN_EINVAL, "%s: null weight / codes / scales", who);
  if (stride < 0 || matrix_stride < 0) return fail(LUTKAN_ESHAPE, "%s: negative stride", who);
  QuantiseArgs a;
  a.w = static_cast<const unsigned char *>(weight); a.codes = static_cast<unsigned char *>(codes); a.scales = scales;
  a.w_stride = stride; a.w_matrix_stride = matrix_stride; a.n = n; a.k = k;
  const int64_t per_matrix = scale_blocks(n) * scale_blocks(k);
  if (matrices > 0x7fffffff / per_matrix) return fail(LUTKAN_EUNSUPPORTED, "%s: too many blocks", who);
  const int64_t all = matrices * per_matrix, launch_blocks = lutkan::kMaxLaunchThreads / 256;      // (more blocks: more launches)
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  for (int64_t first = 0; first < all; first += launch_blocks) {
    a.first = (unsigned)first;
    const dim3 groups((unsigned)std::min(all - first, launch_blocks));
    switch (type) {
      case LUTKAN_F32: hipLaunchKernelGGL(lutkan_quantise_fp8_kernel<LUTKAN_F32>, groups, dim3(256), 0, s, a); break;
      case LUTKAN_F16: hipLaunchKernelGGL(lutkan_quantise_fp8_kernel<LUTKAN_F16>, groups, dim3(256), 0, s, a); break;
      default: hipLaunchKernelGGL(lutkan_quantise_fp8_kernel<LUTKAN_BF16>, groups, dim3(256), 0, s, a); break;
    }
    if (int rc = check_launch(who)) return rc;
  }
  return LUTKAN_OK;
}
