// Conversion to 8-bit integers with a scale for each row, plain (the outputs of a weight, tokens) and after the residual's addition and the
// root-mean-square norm.
#include "lutkan_fp8.h"

namespace {

constexpr float kLargestCode = 127.0f;
constexpr float kSmallestScale = 0x1p-126f;       // a normal number, as is its reciprocal, for a row of zeros too

// Arguments of at most 112 bytes, as of all launches here (a longer one costs the host 0.7 us more): strides travel in 32 bits.
struct RowArgs {
  const unsigned char *x, *residual, *weight;
  unsigned char *residual_out, *codes;
  float *scales;
  int64_t rows;
  int32_t x_stride, residual_stride, residual_out_stride, codes_stride, scales_stride;
  int32_t width, row_waves;
  float eps, inverse_width;
  int32_t weight_type;
};
static_assert(sizeof(RowArgs) <= 112, "launch");

constexpr int kNoResidual = -1, kRowsOfGroup = 4;

// A row's scale from the largest magnitude in it (as bits): NaN for a row that holds a NaN or an infinity.
__device__ __forceinline__ float row_scale(unsigned largest) {
  const float m = __uint_as_float(largest);
  return !finite(m) ? __uint_as_float(0x7fc00000u) : fmaxf(m / kLargestCode, kSmallestScale);
}

// Eight codes: the quotient rounded once (see quotient), then to a whole number, ties to even, by an addition that leaves the number in the low
// bits; those of a NaN are zeros.  |v / scale| is at most 127 (1 + 2^-23).
__device__ __forceinline__ u32x2 whole8(const float (&v)[8], float scale, float inverse) {
  u32x2 c;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    unsigned b[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float q = quotient(v[4 * h + e], scale, inverse);
      b[e] = q == q ? __float_as_uint(q + 12582912.0f) & 0xffu : 0u;
    }
    c[h] = b[0] | (b[1] << 8) | (b[2] << 16) | (b[3] << 24);
  }
  return c;
}

__device__ __forceinline__ void store_codes(unsigned char *codes, int col, int width, u32x2 c) {
  if (col + 8 <= width) { store_any(codes + col, c); return; }
#pragma unroll
  for (int e = 0; e < 8; ++e) if (col + e < width) codes[col + e] = (unsigned char)(c[e >> 2] >> ((e & 3) * 8));
}

template <int TYPE>
__device__ __forceinline__ void read8(const unsigned char *row, int col, int width, float (&v)[8]) {
  if (col + 8 <= width) { values8<TYPE>(load_raw8<TYPE>(row + (size_t)col * type_bytes(TYPE)), v); return; }
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = col + e < width ? load_one<TYPE>(row + (size_t)(col + e) * type_bytes(TYPE)) : 0.0f;
}
__device__ __forceinline__ void read8_of(int type, const unsigned char *row, int col, int width, float (&v)[8]) {
  if (type == LUTKAN_F32) read8<LUTKAN_F32>(row, col, width, v);
  else if (type == LUTKAN_F16) read8<LUTKAN_F16>(row, col, width, v);
  else read8<LUTKAN_BF16>(row, col, width, v);
}

// One row by `row_waves` waves, 64 * 8 * CH columns each; a work-group holds one row, or (row_waves = 1) four.  Every element is read once and
// stays in a register as fp32; lane l of a row's lanes holds the eight columns 8 (l + lanes c), c < CH.
// NORM: the codes do not depend on the norm, the scale does, so that one reduction gives the sum of squares and the largest |h weight|
// together.  Where either leaves fp32's range the row is summed again with a power of 2 on h, and the norm applied before the product.
// Bound by memory: 32768 rows of 1024 (bf16, residual bf16), four bytes read to three written, 43 us replayed, 5.4 TB/s; a copy reaches 4.7 - 5.2, an addition of two
// tensors (two read to one written) 6.0.  One row of 1024: 3.0, of which a launch
// 2.4; 2400 rows of 200 (fp32, no norm) 3.2.
template <int X, int R, int CH, bool NORM>
__global__ __launch_bounds__(1024) void lutkan_int8_rows_kernel(const RowArgs a) {
  const int row_waves = a.row_waves;
  __shared__ float s_sum[16];
  __shared__ unsigned s_largest[16];
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
      float v[8];
      if (col + 8 <= a.width) {
        values8<X>(rx[c], h[c]);
        if constexpr (R != kNoResidual) values8<R>(rr[c], v);
      } else {                                                   // the row ends inside these eight columns, or before them
        read8<X>(x, col, a.width, h[c]);
        if constexpr (R != kNoResidual) read8<R>(r, col, a.width, v);
      }
      if constexpr (R != kNoResidual)
#pragma unroll
        for (int e = 0; e < 8; ++e) h[c][e] += v[e];
    }
  }
  // The row's sum and largest magnitude over its waves.
  const auto reduce = [&](float &sum, unsigned &largest, bool again) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
      if constexpr (NORM) sum += __shfl_xor(sum, off);
      largest = max(largest, (unsigned)__shfl_xor((int)largest, off));
    }
    if (row_waves > 1) {
      if (again) __syncthreads();                                // all have read the first ones
      if (lane == 0) { s_sum[wave] = sum; s_largest[wave] = largest; }
      __syncthreads();
      sum = 0.0f; largest = 0;
      for (int w = 0; w < row_waves; ++w) { sum += s_sum[w]; largest = max(largest, s_largest[w]); }
    }
  };
  float sum = 0.0f, inverse_rms = 1.0f, factor = 1.0f;
  unsigned largest = 0;
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    float weight[8];
    if constexpr (NORM) read8_of(a.weight_type, a.weight, 8 * (at + lanes * c), a.width, weight);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if constexpr (NORM) sum = fmaf(h[c][e], h[c][e], sum);
      largest = max(largest, magnitude(NORM ? h[c][e] * weight[e] : h[c][e]));
    }
  }
  reduce(sum, largest, false);
  bool ordinary = true;
  if constexpr (NORM) {
    const float mean = fmaf(sum, a.inverse_width, a.eps);
    inverse_rms = 1.0f / sqrtf(mean);
    ordinary = finite(sum) && mean >= 0x1p-100f && finite(__uint_as_float(largest)) && __uint_as_float(largest) >= 0x1p-100f;
    if (ordinary) {
      largest = __float_as_uint(__uint_as_float(largest) * inverse_rms);
    } else {
      // (A largest of zero comes here too, and stays zero.)  The largest |h| squared is 2^96 at 2^-80, the smallest that can bring a row here for its
      // squares 2^-24; a sum that is too small was below 2^-85, now 2^115.
      if (!(finite(sum) && mean >= 0x1p-100f)) {
        factor = finite(sum) ? 0x1p100f : 0x1p-80f;
        sum = 0.0f;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
          for (int e = 0; e < 8; ++e) sum = fmaf(h[c][e] * factor, h[c][e] * factor, sum);
        unsigned none = 0;
        reduce(sum, none, true);
        inverse_rms = 1.0f / sqrtf(fmaf(sum, a.inverse_width, a.eps * factor * factor));
      }
      largest = 0;
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        float weight[8];
        const int col = 8 * (at + lanes * c);
        read8_of(a.weight_type, a.weight, col, a.width, weight);
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (col + e < a.width) largest = max(largest, magnitude(h[c][e] * factor * inverse_rms * weight[e]));      // (0 * an infinite norm beyond the row's end is none of its values)
      }
      float none = 0.0f;
      reduce(none, largest, true);
    }
  }
  const float scale = row_scale(largest), inverse = 1.0f / scale;
  if (at == 0) a.scales[row * a.scales_stride] = scale;
  unsigned char *codes = a.codes + row * a.codes_stride;
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const int col = 8 * (at + lanes * c);
    if (col >= a.width) continue;
    float y[8];
    if constexpr (NORM) {
      float weight[8];
      read8_of(a.weight_type, a.weight, col, a.width, weight);
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = ordinary ? h[c][e] * weight[e] * inverse_rms : h[c][e] * factor * inverse_rms * weight[e];
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = h[c][e];
    }
    store_codes(codes, col, a.width, whole8(y, scale, inverse));
    if constexpr (R != kNoResidual) {
      unsigned char *out = a.residual_out + row * a.residual_out_stride * type_bytes(R);
      if (col + 8 <= a.width) {
        store8<R>(out + (size_t)col * type_bytes(R), h[c]);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) if (col + e < a.width) store_one<R>(out + (size_t)(col + e) * type_bytes(R), h[c][e]);
      }
    }
  }
}

// Rows that do not fit the registers of a work-group: read twice, the second time from a cache.
template <int X>
__global__ __launch_bounds__(1024) void lutkan_int8_long_rows_kernel(const RowArgs a) {
  __shared__ unsigned s_largest[16];
  const int64_t row = blockIdx.x;
  const unsigned char *x = a.x + row * a.x_stride * type_bytes(X);
  unsigned largest = 0;
  for (int col = 8 * (int)threadIdx.x; col < a.width; col += 8192) {
    float v[8];
    read8<X>(x, col, a.width, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) largest = max(largest, magnitude(v[e]));
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) largest = max(largest, (unsigned)__shfl_xor((int)largest, off));
  if ((threadIdx.x & 63) == 0) s_largest[threadIdx.x >> 6] = largest;
  __syncthreads();
  largest = 0;
  for (int w = 0; w < 16; ++w) largest = max(largest, s_largest[w]);
  const float scale = row_scale(largest), inverse = 1.0f / scale;
  if (threadIdx.x == 0) a.scales[row * a.scales_stride] = scale;
  for (int col = 8 * (int)threadIdx.x; col < a.width; col += 8192) {
    float v[8];
    read8<X>(x, col, a.width, v);
    store_codes(a.codes + row * a.codes_stride, col, a.width, whole8(v, scale, inverse));
  }
}

constexpr int kMostHeld = 32768;                                 // columns that a work-group's registers hold

// Waves to a row, and their chunks of 512 columns: one wave while the launch fills the GPU with a wave a row and the row fits its registers;
// else enough for eight columns a lane, so that a few rows are spread over many lanes.
struct RowPlan { int waves, chunks; };
RowPlan plan_rows(int64_t rows, int width) {
  int waves = (width + 511) / 512, chunks = 1;
  if (rows >= 2048 && waves <= 4) { chunks = waves; waves = 1; }
  else if (rows >= 1024 && waves <= 16) { chunks = waves > 8 ? 4 : waves > 4 ? 2 : 1; waves = (waves + chunks - 1) / chunks; }
  while (waves > 16) { chunks *= 2; waves = (width + 512 * chunks - 1) / (512 * chunks); }
  return {waves, chunks};
}

template <int X, int R, bool NORM>
void launch_rows_as(const RowArgs &a, int chunks, unsigned groups, unsigned threads, hipStream_t s) {
  switch (chunks) {
    case 1: hipLaunchKernelGGL((lutkan_int8_rows_kernel<X, R, 1, NORM>), dim3(groups), dim3(threads), 0, s, a); break;
    case 2: hipLaunchKernelGGL((lutkan_int8_rows_kernel<X, R, 2, NORM>), dim3(groups), dim3(threads), 0, s, a); break;
    default: hipLaunchKernelGGL((lutkan_int8_rows_kernel<X, R, 4, NORM>), dim3(groups), dim3(threads), 0, s, a); break;
  }
}

template <int X>
int launch_rows_of(RowArgs a, bool norm, int residual_type, const char *who, hipStream_t s) {
  const bool held = a.width <= kMostHeld;
  const RowPlan plan = held ? plan_rows(a.rows, a.width) : RowPlan{16, 0};
  a.row_waves = plan.waves;
  const unsigned threads = plan.waves == 1 ? 64u * kRowsOfGroup : (unsigned)plan.waves * 64u;
  const int group_rows = plan.waves == 1 ? kRowsOfGroup : 1;
  const int64_t launch_rows = lutkan::kMaxLaunchThreads / threads * group_rows, rows = a.rows;      // (more rows: more launches)
  const int64_t residual_bytes = a.residual ? type_bytes(residual_type) : 0;
  for (int64_t first = 0; first < rows; first += launch_rows) {
    a.rows = std::min(rows - first, launch_rows);
    const unsigned groups = (unsigned)((a.rows + group_rows - 1) / group_rows);
    if (!held) hipLaunchKernelGGL(lutkan_int8_long_rows_kernel<X>, dim3(groups), dim3(threads), 0, s, a);
    else if (!norm) launch_rows_as<X, kNoResidual, false>(a, plan.chunks, groups, threads, s);
    else if (!a.residual) launch_rows_as<X, kNoResidual, true>(a, plan.chunks, groups, threads, s);
    else if (residual_type == LUTKAN_F32) launch_rows_as<X, LUTKAN_F32, true>(a, plan.chunks, groups, threads, s);
    else if (residual_type == LUTKAN_F16) launch_rows_as<X, LUTKAN_F16, true>(a, plan.chunks, groups, threads, s);
    else launch_rows_as<X, LUTKAN_BF16, true>(a, plan.chunks, groups, threads, s);
    if (int rc = check_launch(who)) return rc;
    a.x += launch_rows * a.x_stride * type_bytes(X);
    if (a.residual) {
      a.residual += launch_rows * a.residual_stride * residual_bytes;
      a.residual_out += launch_rows * a.residual_out_stride * residual_bytes;
    }
    a.codes += launch_rows * a.codes_stride;
    a.scales += launch_rows * a.scales_stride;
  }
  return LUTKAN_OK;
}

int launch_rows(const RowArgs &a, int type, bool norm, int residual_type, const char *who, hipStream_t s) {
  switch (type) {
    case LUTKAN_F32: return launch_rows_of<LUTKAN_F32>(a, norm, residual_type, who, s);
    case LUTKAN_F16: return launch_rows_of<LUTKAN_F16>(a, norm, residual_type, who, s);
    default: return launch_rows_of<LUTKAN_BF16>(a, norm, residual_type, who, s);
  }
}

}  // namespace

extern "C" int lutkan_rmsnorm_int8(const lutkan_rmsnorm_fp8_args *p, void *hip_stream) {
  const char *who = "lutkan_rmsnorm_int8";
  if (!p) return fail(LUTKAN_EINVAL, "%s: null arguments", who);
  if (p->rows < 0 || p->width < 1) return fail(LUTKAN_EINVAL, "%s: rows %lld, width %d", who, (long long)p->rows, p->width);
  if (p->width > LUTKAN_FP8_MAX_WIDTH) return fail(LUTKAN_EUNSUPPORTED, "%s: width %d, at most %d", who, p->width, LUTKAN_FP8_MAX_WIDTH);
  if (!is_type(p->x_type) || !is_type(p->weight_type) || (p->residual && !is_type(p->residual_type))) return fail(LUTKAN_EINVAL, "%s: bad type", who);
  if (!(p->eps >= 0.0f)) return fail(LUTKAN_EINVAL, "%s: eps must be >= 0", who);
  if (p->rows == 0) return LUTKAN_OK;
  if (!p->x || !p->weight || !p->codes || !p->scales) return fail(LUTKAN_EINVAL, "%s: null x / weight / codes / scales", who);
  if ((p->residual != nullptr) != (p->residual_out != nullptr)) return fail(LUTKAN_EINVAL, "%s: residual and residual_out come together", who);
  if (p->codes_stride < p->width || p->scales_stride < 1 || (p->residual && p->residual_out_stride < p->width))
    return fail(LUTKAN_ESHAPE, "%s: a row of the outputs is longer than its stride", who);
  if (p->x_stride < 0 || (p->residual && p->residual_stride < 0)) return fail(LUTKAN_ESHAPE, "%s: negative stride", who);
  if (std::max({p->x_stride, p->codes_stride, p->scales_stride, p->residual ? p->residual_stride : 0, p->residual ? p->residual_out_stride : 0}) > INT32_MAX)
    return fail(LUTKAN_EUNSUPPORTED, "%s: row strides of at most 2^31 - 1", who);
  RowArgs a{};
  a.x = static_cast<const unsigned char *>(p->x); a.residual = static_cast<const unsigned char *>(p->residual);
  a.weight = static_cast<const unsigned char *>(p->weight); a.residual_out = static_cast<unsigned char *>(p->residual_out);
  a.codes = static_cast<unsigned char *>(p->codes); a.scales = p->scales;
  a.rows = p->rows; a.width = p->width; a.weight_type = p->weight_type; a.eps = p->eps; a.inverse_width = 1.0f / (float)p->width;
  a.x_stride = (int32_t)p->x_stride; a.codes_stride = (int32_t)p->codes_stride; a.scales_stride = (int32_t)p->scales_stride;
  if (p->residual) { a.residual_stride = (int32_t)p->residual_stride; a.residual_out_stride = (int32_t)p->residual_out_stride; }
  return launch_rows(a, p->x_type, true, p->residual_type, who, static_cast<hipStream_t>(hip_stream));
}

extern "C" int lutkan_quantise_int8(const void *rows, int32_t type, int64_t matrices, int32_t n, int32_t k, int64_t stride, int64_t matrix_stride,
                                    void *codes, float *scales, void *hip_stream) {
  const char *who = "lutkan_quantise_int8";
  if (!is_type(type)) return fail(LUTKAN_EINVAL, "%s: bad type", who);
  if (matrices < 0 || n < 0 || k < 1) return fail(LUTKAN_EINVAL, "%s: %lld matrices of %d x %d", who, (long long)matrices, n, k);
  if (k > LUTKAN_INT8_MAX_INPUTS) return fail(LUTKAN_EUNSUPPORTED, "%s: rows of %d, at most %d", who, k, LUTKAN_INT8_MAX_INPUTS);
  if (matrices == 0 || n == 0) return LUTKAN_OK;
  if (!rows || !codes || !scales) return fail(LUTKAN_EINVAL, "%s: null rows / codes / scales", who);
  if (stride < 0 || matrix_stride < 0) return fail(LUTKAN_ESHAPE, "%s: negative stride", who);
  if (stride > INT32_MAX) return fail(LUTKAN_EUNSUPPORTED, "%s: row strides of at most 2^31 - 1", who);
  RowArgs a{};
  a.x = static_cast<const unsigned char *>(rows); a.codes = static_cast<unsigned char *>(codes); a.scales = scales;
  a.width = k; a.x_stride = (int32_t)stride; a.codes_stride = k; a.scales_stride = 1;
  // Matrices that follow each other at the distance of their rows are one, and so are those of a single row.
  const bool single = n == 1 && matrix_stride <= INT32_MAX;
  const bool one = single || matrices == 1 || (matrix_stride == (int64_t)n * stride && matrices <= INT64_MAX / n / (int64_t)(4 * std::max<int64_t>(stride, k)));
  if (single && matrices > 1) a.x_stride = (int32_t)matrix_stride;
  a.rows = one ? matrices * n : n;
  for (int64_t m = 0; m < (one ? 1 : matrices); ++m) {
    if (int rc = launch_rows(a, type, false, 0, who, static_cast<hipStream_t>(hip_stream))) return rc;
    a.x += matrix_stride * type_bytes(type); a.codes += (int64_t)n * k; a.scales += n;
  }
  return LUTKAN_OK;
}
