// A mixture of experts around the products by expert: a router's choices sorted by expert, and the experts' rows back in the tokens' order,
// weighted, with the gradients.
#include "lutkan_fp8.h"

namespace {

__device__ __forceinline__ int64_t whole_number(const void *p, int64_t at, int bytes) {
  return bytes == 8 ? static_cast<const int64_t *>(p)[at] : static_cast<const int32_t *>(p)[at];
}

// ---- sort ----------------------------------------------------------------------------------------------------------
// Choices are sorted by expert in one pass of a counting sort where there are few experts, and by the low, then the high bits of the expert where there
// are more than its counters hold.
struct SortArgs {
  const void *expert;
  int32_t *rows, *places, *group_sizes;                           // nullable: of another pass, resp. counted from the sorted experts
  const int32_t *order;                                           // the choices as the pass before left them; nullable: as they are
  int32_t *order_out, *sorted;                                    // the pass's order, the sorted choices' experts; nullable
  int32_t *counts;                                                // [work-group][bins], several work-groups
  int64_t stride;
  int32_t choices, top, experts, bins;
  int32_t segment;                                                // choices of a wave, a multiple of 64
  int8_t expert_bytes, shift;                                     // a bin: the bits of the expert from here on
};
static_assert(sizeof(SortArgs) <= 112, "launch");

constexpr int kSortWaves = 16;
// Chunks of 64 choices whose experts a wave holds; their loop is unrolled, and a longer code costs more to fetch than it saves (with 16 of them 524288 choices take
// 16.2 us for 11.9, one token 3.9 for 3.3).
constexpr int kSortHeld = 4;
// Choices of one work-group's launch: 4080 of 64 experts take 7.8 us and 4800 10.2, two launches of several work-groups 8.4 for these.
constexpr int kSortSingle = 64 * kSortHeld * kSortWaves;
constexpr int kSortDigit = 11, kSortBins = (1 << kSortDigit) + 1; // (2048 experts and the dropped ones)

// The expert of choice c, `experts` for a choice that is dropped.
__device__ __forceinline__ int expert_of(const SortArgs &a, int c) {
  const int64_t at = a.stride == a.top ? c : c / a.top * a.stride + c % a.top;
  const int64_t e = whole_number(a.expert, at, a.expert_bytes);
  return e >= 0 && e < a.experts ? (int)e : a.experts;
}
// (One pass: all bits.)
__device__ __forceinline__ int bin_of(const SortArgs &a, int expert) { return a.bins == 1 << kSortDigit ? (expert >> a.shift) & (a.bins - 1) : expert; }

// Lanes with the same bin as the own one, among those that hold a choice.
__device__ __forceinline__ unsigned long long same_bin(int bin, int bits, bool held) {
  unsigned long long same = __ballot(held);
  for (int b = 0; b < bits; ++b) {
    const unsigned long long set = __ballot((bin >> b) & 1);
    same &= (bin >> b) & 1 ? set : ~set;
  }
  return same;
}

// A wave's choices of kSortHeld chunks of 64: which ones, and their experts, all asked for at once.
struct SortHeld {
  int choice[kSortHeld], expert[kSortHeld];
  __device__ __forceinline__ void read(const SortArgs &a, int first, int last) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int k = 0; k < kSortHeld; ++k) {
      const int i = first + 64 * k + lane;
      choice[k] = a.order && i < last ? a.order[i] : i;
    }
#pragma unroll
    for (int k = 0; k < kSortHeld; ++k) {
      const int i = first + 64 * k + lane;
      expert[k] = i < last ? expert_of(a, choice[k]) : 0;
    }
  }
};

// How many choices of each bin the work-group's waves hold, into s_count [wave][bins], which is zero.  `held`: the first chunks; it keeps the last.
__device__ __forceinline__ void count_bins(const SortArgs &a, int *s_count, SortHeld &held, int first, int last, int wave) {
  for (int at = first; at < last; at += 64 * kSortHeld) {
    if (at != first) held.read(a, at, last);
#pragma unroll
    for (int k = 0; k < kSortHeld; ++k)
      if (at + 64 * k + (int)(threadIdx.x & 63) < last) atomicAdd(&s_count[wave * a.bins + bin_of(a, held.expert[k])], 1);
  }
}

__global__ __launch_bounds__(64 * kSortWaves) void lutkan_expert_count_kernel(const SortArgs a) {
  extern __shared__ int s_count[];
  const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const int64_t begin = ((int64_t)blockIdx.x * waves + wave) * a.segment;
  const int first = (int)min(begin, (int64_t)a.choices), last = (int)min(begin + a.segment, (int64_t)a.choices);
  SortHeld held;
  held.read(a, first, last);
  for (int i = threadIdx.x; i < waves * a.bins; i += blockDim.x) s_count[i] = 0;
  __syncthreads();
  count_bins(a, s_count, held, first, last, wave);
  __syncthreads();
  for (int e = threadIdx.x; e < a.bins; e += blockDim.x) {
    int sum = 0;
    for (int w = 0; w < waves; ++w) sum += s_count[w * a.bins + e];
    a.counts[(int64_t)blockIdx.x * a.bins + e] = sum;
  }
}

// A counting sort: the place of a choice is the number of choices of lower bins, of its bin in work-groups and waves before its own, and before it
// in its wave.  The last comes from ballots over the bits of the bin, so that equal bins keep their order and no atomic decides it (the atomics
// here count).  Bound by latencies: launches, a chain of loads, counts and scans: one token's 2 choices 2.7 us (a launch alone 2.4), 524288 choices of 64 experts
// 3.6 + 9.8, where their bytes take 1.6.  Two passes: of 4096 experts 120 us, where 2048 take 41.
template <bool SEVERAL>
__global__ __launch_bounds__(64 * kSortWaves) void lutkan_expert_sort_kernel(const SortArgs a) {
  extern __shared__ int s_count[];                                // [waves][bins], then the bins' totals, later first places, the waves' sums, the bins' counts before
  const int bins = a.bins, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  int *s_total = s_count + waves * bins, *s_wave = s_total + bins, *s_before = s_wave + kSortWaves;
  const int64_t begin = ((int64_t)blockIdx.x * waves + wave) * a.segment;
  const int first = (int)min(begin, (int64_t)a.choices), last = (int)min(begin + a.segment, (int64_t)a.choices);
  SortHeld held;
  held.read(a, first, last);
  for (int i = threadIdx.x; i < waves * bins; i += blockDim.x) s_count[i] = 0;
  if constexpr (SEVERAL)
    for (int e = threadIdx.x; e < bins; e += blockDim.x) s_total[e] = s_before[e] = 0;
  __syncthreads();
  if constexpr (SEVERAL) {                                        // the work-groups' counts, while the choices are on their way: as many threads to a bin as there are
    const int parts = max(1, (int)blockDim.x / bins), part = threadIdx.x / bins;
    for (int e = parts > 1 ? threadIdx.x % bins : threadIdx.x; e < bins && part < parts; e += parts > 1 ? bins : blockDim.x) {
      int before = 0, total = 0;
#pragma unroll 8
      for (int g = parts > 1 ? part : 0; g < (int)gridDim.x; g += parts) {
        const int n = a.counts[(int64_t)g * bins + e];
        before += g < (int)blockIdx.x ? n : 0;
        total += n;
      }
      atomicAdd(&s_before[e], before);
      atomicAdd(&s_total[e], total);
    }
  }
  count_bins(a, s_count, held, first, last, wave);
  __syncthreads();
  // Every bin: in place of the waves' counts, how many of it lie before each wave.
  for (int e = threadIdx.x; e < bins; e += blockDim.x) {
    int before = SEVERAL ? s_before[e] : 0;
    for (int w = 0; w < waves; ++w) {
      const int n = s_count[w * bins + e];
      s_count[w * bins + e] = before;
      before += n;
    }
    if constexpr (!SEVERAL) s_total[e] = before;
  }
  __syncthreads();
  // The bins' first places: sums of runs of bins, a run to a thread, then the run itself.
  const int run = (bins + blockDim.x - 1) / blockDim.x, run_first = min((int)threadIdx.x * run, bins), run_last = min(run_first + run, bins);
  int sum = 0;
  for (int e = run_first; e < run_last; ++e) sum += s_total[e];
  int with = sum;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int v = __shfl_up(with, off);
    with += lane >= off ? v : 0;
  }
  if (lane == 63) s_wave[wave] = with;
  __syncthreads();
  int at = with - sum;
  for (int w = 0; w < wave; ++w) at += s_wave[w];
  for (int e = run_first; e < run_last; ++e) {
    const int n = s_total[e];
    if (a.group_sizes && blockIdx.x == 0 && e < a.experts) a.group_sizes[e] = n;
    s_total[e] = at;
    at += n;
  }
  __syncthreads();
  const int bits = 32 - __builtin_clz(bins - 1);                  // (bins >= 2)
  const bool again = last - first > 64 * kSortHeld;               // (the chunks that are held are the last)
  for (int i0 = first; i0 < last; i0 += 64 * kSortHeld) {
    if (again) held.read(a, i0, last);
#pragma unroll
    for (int k = 0; k < kSortHeld; ++k) {
      if (i0 + 64 * k >= last) break;
      const bool here = i0 + 64 * k + lane < last;
      const int c = held.choice[k], expert = held.expert[k], bin = bin_of(a, expert);
      const unsigned long long same = same_bin(bin, bits, here);
      const int rank = __popcll(same & ((1ull << lane) - 1));
      if (here) {
        const int place = s_total[bin] + s_count[wave * bins + bin] + rank;
        const bool is_held = expert < a.experts;
        if (a.rows) {
          a.rows[place] = is_held ? c / a.top : -1;
          a.places[c] = is_held ? place : -1;
        }
        if (a.order_out) a.order_out[place] = c;
        if (a.sorted) a.sorted[place] = expert;
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");    // all lanes have read the count before its first lane raises it
      if (here && rank == 0) s_count[wave * bins + bin] += __popcll(same);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
  }
}

// How many of the sorted experts are below e.
__device__ __forceinline__ int below(const int32_t *sorted, int n, int e) {
  int low = 0, high = n;
  while (low < high) {
    const int mid = low + (high - low) / 2;
    if (sorted[mid] < e) low = mid + 1;
    else high = mid;
  }
  return low;
}
__global__ __launch_bounds__(256) void lutkan_expert_sizes_kernel(const int32_t *sorted, int32_t choices, int32_t experts, int32_t *group_sizes) {
  const int e = blockIdx.x * 256 + threadIdx.x;
  if (e < experts) group_sizes[e] = below(sorted, choices, e + 1) - below(sorted, choices, e);
}

// Waves of a work-group and choices of a wave: one work-group up to kSortSingle choices, else at most 256 work-groups.
struct SortPlan {
  int waves, segment, groups, bins;
  bool one_pass;
  size_t count_words, words;                                      // of the workspace: counts, then the two orders
};
SortPlan plan_sort(int64_t choices, int experts) {
  SortPlan p;
  const int64_t chunks = (choices + 63) / 64;
  if (choices <= kSortSingle) {
    p.waves = (int)std::max<int64_t>(1, std::min<int64_t>(chunks, kSortWaves));
    p.segment = (int)((chunks + p.waves - 1) / p.waves * 64);
    p.groups = 1;
  } else {
    // More work-groups are shorter, and each reads the counts of all: 524288 choices of 256 experts take 21.2 us with 81 of them, 16.9 with 160; of 64
    // experts 17.5, 13.3 and 12.5 with 112, 160 and 256.
    const double best = std::sqrt(800.0 * (double)chunks / std::min(experts + 1, 1 << kSortDigit));
    const int64_t most = (int64_t)kSortWaves * std::max(1, (int)std::min(best, 256.0)), of_wave = (chunks + most - 1) / most;
    p.waves = kSortWaves;
    p.segment = (int)(of_wave * 64);
    p.groups = (int)((chunks + of_wave * kSortWaves - 1) / (of_wave * kSortWaves));
  }
  p.one_pass = experts < kSortBins;
  p.bins = p.one_pass ? experts + 1 : 1 << kSortDigit;
  p.count_words = p.groups > 1 ? (size_t)p.groups * p.bins : 0;
  p.words = p.count_words + (p.one_pass ? 0 : 2 * (size_t)choices);
  return p;
}

int launch_sort(const SortArgs &a, const SortPlan &p, const char *who, hipStream_t s) {
  static LdsCap caps[3];
  const size_t counts = (size_t)p.waves * p.bins * sizeof(int), lds = counts + ((size_t)p.bins * (p.groups > 1 ? 2 : 1) + kSortWaves) * sizeof(int);
  const bool more = lds > 64 * 1024;                              // (below that no kernel's cap has to be raised)
  if (p.groups == 1) {
    if (int rc = more ? raise_lds_cap(lutkan_expert_sort_kernel<false>, &caps[0], who) : LUTKAN_OK) return rc;
    hipLaunchKernelGGL(lutkan_expert_sort_kernel<false>, dim3(1), dim3(64 * p.waves), lds, s, a);
    return check_launch(who);
  }
  if (int rc = more ? raise_lds_cap(lutkan_expert_count_kernel, &caps[1], who) : LUTKAN_OK) return rc;
  if (int rc = more ? raise_lds_cap(lutkan_expert_sort_kernel<true>, &caps[2], who) : LUTKAN_OK) return rc;
  hipLaunchKernelGGL(lutkan_expert_count_kernel, dim3(p.groups), dim3(64 * p.waves), counts, s, a);
  if (int rc = check_launch(who)) return rc;
  hipLaunchKernelGGL(lutkan_expert_sort_kernel<true>, dim3(p.groups), dim3(64 * p.waves), lds, s, a);
  return check_launch(who);
}

// ---- combine -------------------------------------------------------------------------------------------------------
struct CombineArgs {
  const unsigned char *y, *weights;
  const void *places;
  unsigned char *out;
  int64_t y_stride, out_stride, y_rows, tokens;
  int32_t top, width, weights_type, places_bytes;
};
static_assert(sizeof(CombineArgs) <= 112, "launch");

__device__ __forceinline__ float weight_at(const unsigned char *weights, int type, int64_t at) {
  const unsigned char *p = weights + at * type_bytes(type);
  return type == LUTKAN_F32 ? load_one<LUTKAN_F32>(p) : type == LUTKAN_F16 ? load_one<LUTKAN_F16>(p) : load_one<LUTKAN_BF16>(p);
}
__device__ __forceinline__ void store_weight(unsigned char *weights, int type, int64_t at, float v) {
  unsigned char *p = weights + at * type_bytes(type);
  if (type == LUTKAN_F32) store_one<LUTKAN_F32>(p, v);
  else if (type == LUTKAN_F16) store_one<LUTKAN_F16>(p, v);
  else store_one<LUTKAN_BF16>(p, v);
}

// Eight columns of a row from col on, zeros behind its end.
template <int TYPE>
__device__ __forceinline__ void read8(const unsigned char *row, int col, int width, float (&v)[8]) {
  if (col + 8 <= width) { values8<TYPE>(load_raw8<TYPE>(row + (size_t)col * type_bytes(TYPE)), v); return; }
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = col + e < width ? load_one<TYPE>(row + (size_t)(col + e) * type_bytes(TYPE)) : 0.0f;
}
template <int TYPE>
__device__ __forceinline__ void write8(unsigned char *row, int col, int width, const float (&v)[8]) {
  if (col + 8 <= width) { store8<TYPE>(row + (size_t)col * type_bytes(TYPE), v); return; }
#pragma unroll
  for (int e = 0; e < 8; ++e) if (col + e < width) store_one<TYPE>(row + (size_t)(col + e) * type_bytes(TYPE), v[e]);
}

typedef unsigned int u32x4_any __attribute__((ext_vector_type(4), aligned(2)));        // at any address that an element can have

// Eight columns as they lie in memory, asked for and used later; a row that ends inside them is read element by element.  ONCE: nobody else reads the row,
// and it need not stay in the caches (16384 tokens of four rows of 2048, bf16: joined in 66 -> 60 us, gradients 118 -> 99; of rows that several read 43 -> 49).
template <int TYPE>
struct Asked8 {
  Raw8<TYPE> raw;
  template <bool ONCE>
  __device__ __forceinline__ void ask(const unsigned char *row, int col, int width) {
    if (col + 8 > width) return;
    const u32x4_any *p = reinterpret_cast<const u32x4_any *>(row + (size_t)col * type_bytes(TYPE));
#pragma unroll
    for (int h = 0; h < type_bytes(TYPE) / 2; ++h) {
      if constexpr (ONCE) raw.v[h] = __builtin_nontemporal_load(p + h);
      else raw.v[h] = p[h];
    }
  }
  __device__ __forceinline__ void get(const unsigned char *row, int col, int width, float (&v)[8]) const {
    if (col + 8 <= width) values8<TYPE>(raw, v);
    else read8<TYPE>(row, col, width, v);
  }
};

// Up to 64 of a token's choices, one a lane: their rows of y (-1: none) and weights.
struct Choices {
  int row;
  float weight;
  __device__ __forceinline__ Choices(const void *places, int places_bytes, const unsigned char *weights, int weights_type, int64_t token, int top, int first, int64_t y_rows) {
    const int j = first + (int)(threadIdx.x & 63);
    row = -1;
    weight = 1.0f;
    if (j < top) {
      const int64_t place = whole_number(places, token * top + j, places_bytes);
      if (place >= 0 && place < y_rows) row = (int)place;
      if (weights) weight = weight_at(weights, weights_type, token * top + j);
    }
  }
  __device__ __forceinline__ int row_of(int j) const { return __builtin_amdgcn_readlane(row, j); }
  __device__ __forceinline__ float weight_of(int j) const { return __uint_as_float(__builtin_amdgcn_readlane((int)__float_as_uint(weight), j)); }
};

constexpr int kJoined = 4;                                       // rows that are read before the first is used

// A wave sums 512 columns of one token, eight a lane.  ONCE: several rows a token, which no other token has.
// Bound by memory: 16384 tokens of four rows of 2048 (bf16) 60 - 67 us, 5.0 - 5.6 TB/s (an addition of two tensors, two reads to a write: 6.0); 16 tokens of two of 1024 (fp32) 3.0.
template <int Y, int O, bool ONCE>
__global__ __launch_bounds__(256) void lutkan_expert_combine_kernel(const CombineArgs a) {
  const int lane = threadIdx.x & 63, pieces = (a.width + 511) / 512;
  const int64_t unit = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), token = unit / pieces;
  if (token >= a.tokens) return;
  const int col = (int)(unit - token * pieces) * 512 + 8 * lane;
  float sum[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
  for (int first = 0; first < a.top; first += 64) {
    const Choices choices(a.places, a.places_bytes, a.weights, a.weights_type, token, a.top, first, a.y_rows);
    const int count = min(a.top - first, 64);
    for (int j0 = 0; j0 < count; j0 += kJoined) {
      Asked8<Y> asked[kJoined];
#pragma unroll
      for (int j = 0; j < kJoined; ++j) {                        // (lanes behind the last choice hold none)
        const int row = j0 + j < 64 ? choices.row_of(j0 + j) : -1;
        if (row >= 0) asked[j].template ask<ONCE>(a.y + row * a.y_stride * type_bytes(Y), col, a.width);
      }
#pragma unroll
      for (int j = 0; j < kJoined; ++j) {
        const int row = j0 + j < 64 ? choices.row_of(j0 + j) : -1;
        if (row < 0) continue;
        float v[8];
        asked[j].get(a.y + row * a.y_stride * type_bytes(Y), col, a.width, v);
        const float w = choices.weight_of(j0 + j);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] += w * v[e];          // (two roundings, as an elementwise product and a sum have)
      }
    }
  }
  if (col < a.width) write8<O>(a.out + token * a.out_stride * type_bytes(O), col, a.width, sum);
}

struct BackwardArgs {
  const unsigned char *grad, *y, *weights;
  const void *rows, *places;
  unsigned char *grad_y, *grad_weights;
  int32_t y_rows, tokens;
  int32_t grad_stride, y_stride, grad_y_stride;
  int32_t top, width, checks;                                    // checks: work-groups that look for rows without a choice
  int8_t weights_type, rows_bytes, places_bytes;
};
static_assert(sizeof(BackwardArgs) <= 112, "launch");

constexpr int kCheckRows = 16;                                   // rows of y that a wave looks through, four lanes each

// A work-group takes a token: its waves share the columns, and their sums meet in LDS in the waves' order.  The waves of the first work-groups look
// through the rows of y for those that no place leads to.  (64 rows a work-group: the 300 dropped rows of 1000 tokens of three, 300 wide, were all in five of
// them, 23 us for 7.  16 a work-group of four waves, or looked for by the tokens' work-groups: more of them on the GPU at a time, 16384 tokens of four, 2048 wide, 5 - 20 us more.)
// Bound by memory: that case 105 - 110 us, 5.5 - 5.7 TB/s.
template <int G, int Y>
__global__ __launch_bounds__(1024) void lutkan_expert_combine_backward_kernel(const BackwardArgs a) {
  __shared__ float s_sum[16][kJoined];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  if ((int)blockIdx.x < a.checks) {
    const int64_t first = ((int64_t)blockIdx.x * waves + wave) * kCheckRows, row = first + (lane >> 2);
    bool found = row >= a.y_rows;
    if (!found) {
      const int64_t token = whole_number(a.rows, row, a.rows_bytes);
      if (token >= 0 && token < a.tokens)
        for (int j = lane & 3; j < a.top; j += 4) found |= whole_number(a.places, token * a.top + j, a.places_bytes) == row;
    }
    const unsigned long long by_four = __ballot(found);
    const float zeros[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    for (int r = 0; r < kCheckRows; ++r) {
      if (by_four >> (4 * r) & 15) continue;
      for (int col = 8 * lane; col < a.width; col += 512) write8<Y>(a.grad_y + (first + r) * a.grad_y_stride * type_bytes(Y), col, a.width, zeros);
    }
    return;
  }
  const int64_t token = blockIdx.x - a.checks;
  const unsigned char *grad = a.grad + token * a.grad_stride * type_bytes(G);
  for (int first = 0; first < a.top; first += 64) {
    const Choices choices(a.places, a.places_bytes, a.weights, a.weights_type, token, a.top, first, a.y_rows);
    const unsigned long long held = __ballot(choices.row >= 0 && whole_number(a.rows, choices.row, a.rows_bytes) == token);      // (one way and back)
    const int count = min(a.top - first, 64);
    for (int j0 = 0; j0 < count; j0 += kJoined) {
      float dot[kJoined];
      int row[kJoined];
#pragma unroll
      for (int j = 0; j < kJoined; ++j) {
        dot[j] = 0.0f;
        row[j] = j0 + j < 64 && (held >> ((j0 + j) & 63) & 1) ? choices.row_of(j0 + j) : -1;
      }
      for (int col = 8 * (int)threadIdx.x; col < a.width; col += 8 * blockDim.x) {
        Asked8<G> asked;
        Asked8<Y> of_y[kJoined];
        asked.template ask<false>(grad, col, a.width);
        if (a.weights)
#pragma unroll
          for (int j = 0; j < kJoined; ++j) if (row[j] >= 0) of_y[j].template ask<true>(a.y + row[j] * (int64_t)a.y_stride * type_bytes(Y), col, a.width);
        float g[8];
        asked.get(grad, col, a.width, g);
#pragma unroll
        for (int j = 0; j < kJoined; ++j) {
          if (row[j] < 0) continue;
          float v[8];
          if (a.weights) {
            of_y[j].get(a.y + row[j] * (int64_t)a.y_stride * type_bytes(Y), col, a.width, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) dot[j] = fmaf(g[e], v[e], dot[j]);
          }
          const float w = choices.weight_of(j0 + j);
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = g[e] * w;
          write8<Y>(a.grad_y + row[j] * (int64_t)a.grad_y_stride * type_bytes(Y), col, a.width, v);
        }
      }
      if (!a.weights) continue;
#pragma unroll
      for (int j = 0; j < kJoined; ++j)
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) dot[j] += __shfl_xor(dot[j], off);
      if (waves > 1) {
        if (lane == 0)
#pragma unroll
          for (int j = 0; j < kJoined; ++j) s_sum[wave][j] = dot[j];
        __syncthreads();
        if (threadIdx.x < kJoined) {
          float all = 0.0f;
          for (int o = 0; o < waves; ++o) all += s_sum[o][threadIdx.x];
          const int j = j0 + (int)threadIdx.x;
          if (j < count) store_weight(a.grad_weights, a.weights_type, token * a.top + first + j, held >> j & 1 ? all : 0.0f);
        }
        __syncthreads();
      } else {
#pragma unroll
        for (int j = 0; j < kJoined; ++j)
          if (lane == j && j0 + j < count) store_weight(a.grad_weights, a.weights_type, token * a.top + first + j0 + j, row[j] >= 0 ? dot[j] : 0.0f);
      }
    }
  }
}

template <typename F>
void with_types(int first, int second, const F &f) {
  const auto inner = [&](auto one) {
    switch (second) {
      case LUTKAN_F32: f(one, std::integral_constant<int, LUTKAN_F32>()); break;
      case LUTKAN_F16: f(one, std::integral_constant<int, LUTKAN_F16>()); break;
      default: f(one, std::integral_constant<int, LUTKAN_BF16>()); break;
    }
  };
  switch (first) {
    case LUTKAN_F32: inner(std::integral_constant<int, LUTKAN_F32>()); break;
    case LUTKAN_F16: inner(std::integral_constant<int, LUTKAN_F16>()); break;
    default: inner(std::integral_constant<int, LUTKAN_BF16>()); break;
  }
}

constexpr int kMostCounted = 1 << 30;                             // (columns, and a token's choices, are counted in 32 bits, past their end too)

bool is_whole(int bytes) { return bytes == 4 || bytes == 8; }

// What both directions check: the counts and the tokens' rows.
int check_tokens(const char *who, int64_t tokens, int32_t top, int32_t width, int64_t y_rows) {
  if (tokens < 0 || top < 1 || width < 1 || y_rows < 0) return fail(LUTKAN_EINVAL, "%s: %lld tokens, %d each, width %d, %lld rows", who, (long long)tokens, top, width, (long long)y_rows);
  if (width > kMostCounted || top > kMostCounted) return fail(LUTKAN_EUNSUPPORTED, "%s: width %d, %d choices a token, at most %d", who, width, top, kMostCounted);
  if (tokens > INT32_MAX || y_rows > INT32_MAX) return fail(LUTKAN_EUNSUPPORTED, "%s: at most 2^31 - 1 tokens and rows", who);
  return LUTKAN_OK;
}

}  // namespace

extern "C" size_t lutkan_expert_sort_workspace_bytes(int64_t tokens, int32_t top, int32_t experts) {
  if (tokens < 0 || top < 1 || experts < 1 || experts > LUTKAN_EXPERT_MAX || tokens > LUTKAN_EXPERT_MAX_CHOICES / top) return 0;
  return plan_sort(tokens * top, experts).words * sizeof(int32_t);
}

extern "C" int lutkan_expert_sort(const lutkan_expert_sort_args *p, void *hip_stream) {
  const char *who = "lutkan_expert_sort";
  if (!p) return fail(LUTKAN_EINVAL, "%s: null arguments", who);
  if (p->tokens < 0 || p->top < 1 || p->experts < 1) return fail(LUTKAN_EINVAL, "%s: %lld tokens, %d each of %d experts", who, (long long)p->tokens, p->top, p->experts);
  if (p->experts > LUTKAN_EXPERT_MAX) return fail(LUTKAN_EUNSUPPORTED, "%s: %d experts, at most %d", who, p->experts, LUTKAN_EXPERT_MAX);
  if (p->tokens > LUTKAN_EXPERT_MAX_CHOICES / p->top) return fail(LUTKAN_EUNSUPPORTED, "%s: %lld tokens, %d each, at most %d in all", who, (long long)p->tokens, p->top, LUTKAN_EXPERT_MAX_CHOICES);
  if (!is_whole(p->expert_bytes)) return fail(LUTKAN_EINVAL, "%s: expert is whole numbers of 4 or 8 bytes", who);
  if (!p->group_sizes || (p->tokens > 0 && (!p->expert || !p->rows || !p->places))) return fail(LUTKAN_EINVAL, "%s: null expert / rows / places / group_sizes", who);
  if (p->expert_stride < 0 || p->expert_stride > INT64_MAX / 8 / std::max<int64_t>(p->tokens, 1)) return fail(LUTKAN_ESHAPE, "%s: stride", who);
  const size_t needed = lutkan_expert_sort_workspace_bytes(p->tokens, p->top, p->experts);
  if (p->workspace_bytes < needed || (needed && !p->workspace)) return fail(LUTKAN_ESHAPE, "%s: workspace of %zu bytes, needs %zu", who, p->workspace_bytes, needed);
  if (needed && (reinterpret_cast<uintptr_t>(p->workspace) & 3)) return fail(LUTKAN_EINVAL, "%s: workspace must be 4-byte aligned", who);
  const SortPlan plan = plan_sort(p->tokens * p->top, p->experts);
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  SortArgs a{};
  a.expert = p->expert; a.rows = p->rows; a.places = p->places; a.group_sizes = p->group_sizes; a.counts = static_cast<int32_t *>(p->workspace);
  a.stride = p->expert_stride; a.choices = (int32_t)(p->tokens * p->top); a.top = p->top; a.experts = p->experts; a.expert_bytes = (int8_t)p->expert_bytes;
  a.bins = plan.bins; a.segment = plan.segment;
  if (plan.one_pass) return launch_sort(a, plan, who, s);
  int32_t *order = a.counts + plan.count_words, *sorted = order + a.choices;
  a.rows = a.places = a.group_sizes = nullptr;
  a.order_out = order;
  if (int rc = launch_sort(a, plan, who, s)) return rc;
  a.rows = p->rows; a.places = p->places;
  a.order = order; a.order_out = nullptr; a.sorted = sorted; a.shift = kSortDigit;
  if (int rc = launch_sort(a, plan, who, s)) return rc;
  hipLaunchKernelGGL(lutkan_expert_sizes_kernel, dim3((p->experts + 255) / 256), dim3(256), 0, s, sorted, a.choices, p->experts, p->group_sizes);
  return check_launch(who);
}

extern "C" int lutkan_expert_combine(const lutkan_expert_combine_args *p, void *hip_stream) {
  const char *who = "lutkan_expert_combine";
  if (!p) return fail(LUTKAN_EINVAL, "%s: null arguments", who);
  if (int rc = check_tokens(who, p->tokens, p->top, p->width, p->y_rows)) return rc;
  if (!is_type(p->y_type) || !is_type(p->out_type) || (p->weights && !is_type(p->weights_type))) return fail(LUTKAN_EINVAL, "%s: bad type", who);
  if (!is_whole(p->places_bytes)) return fail(LUTKAN_EINVAL, "%s: places are whole numbers of 4 or 8 bytes", who);
  if (p->tokens == 0) return LUTKAN_OK;
  if ((p->y_rows > 0 && !p->y) || !p->places || !p->out) return fail(LUTKAN_EINVAL, "%s: null y / places / out", who);
  if (p->y_stride < 0 || p->out_stride < p->width) return fail(LUTKAN_ESHAPE, "%s: a negative stride, or a row of out that is longer than its stride", who);
  if (p->y_stride > INT32_MAX || p->out_stride > INT32_MAX) return fail(LUTKAN_EUNSUPPORTED, "%s: row strides of at most 2^31 - 1", who);
  CombineArgs a;
  a.y = static_cast<const unsigned char *>(p->y); a.weights = static_cast<const unsigned char *>(p->weights);
  a.y_stride = p->y_stride; a.out_stride = p->out_stride; a.y_rows = p->y_rows;
  a.top = p->top; a.width = p->width; a.weights_type = p->weights_type; a.places_bytes = p->places_bytes;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const int64_t pieces = ((int64_t)p->width + 511) / 512, launch_tokens = lutkan::kMaxLaunchThreads / 256 * 4 / pieces;      // (more tokens: more launches)
  for (int64_t first = 0; first < p->tokens; first += launch_tokens) {
    a.tokens = std::min(p->tokens - first, launch_tokens);
    a.places = static_cast<const unsigned char *>(p->places) + first * p->top * p->places_bytes;
    if (p->weights) a.weights = static_cast<const unsigned char *>(p->weights) + first * p->top * type_bytes(p->weights_type);
    a.out = static_cast<unsigned char *>(p->out) + first * p->out_stride * type_bytes(p->out_type);
    const dim3 groups((unsigned)((a.tokens * pieces + 3) / 4));
    with_types(p->y_type, p->out_type, [&](auto y, auto o) {
      if (p->top > 1) hipLaunchKernelGGL((lutkan_expert_combine_kernel<y, o, true>), groups, dim3(256), 0, s, a);
      else hipLaunchKernelGGL((lutkan_expert_combine_kernel<y, o, false>), groups, dim3(256), 0, s, a);
    });
    if (int rc = check_launch(who)) return rc;
  }
  return LUTKAN_OK;
}

extern "C" int lutkan_expert_combine_backward(const lutkan_expert_combine_backward_args *p, void *hip_stream) {
  const char *who = "lutkan_expert_combine_backward";
  if (!p) return fail(LUTKAN_EINVAL, "%s: null arguments", who);
  if (int rc = check_tokens(who, p->tokens, p->top, p->width, p->y_rows)) return rc;
  if (!is_type(p->grad_type) || !is_type(p->y_type) || (p->weights && !is_type(p->weights_type))) return fail(LUTKAN_EINVAL, "%s: bad type", who);
  if (!is_whole(p->places_bytes) || !is_whole(p->rows_bytes)) return fail(LUTKAN_EINVAL, "%s: rows and places are whole numbers of 4 or 8 bytes", who);
  if ((p->weights != nullptr) != (p->grad_weights != nullptr) && p->tokens > 0) return fail(LUTKAN_EINVAL, "%s: weights and grad_weights come together", who);
  if (p->tokens > 0 && (!p->grad || !p->places)) return fail(LUTKAN_EINVAL, "%s: null grad / places", who);
  if (p->y_rows > 0 && (!p->rows || !p->grad_y || (p->weights && !p->y))) return fail(LUTKAN_EINVAL, "%s: null rows / grad_y / y", who);
  if (p->grad_stride < 0 || (p->weights && p->y_stride < 0) || (p->y_rows > 0 && p->grad_y_stride < p->width)) return fail(LUTKAN_ESHAPE, "%s: a negative stride, or a row of grad_y that is longer than its stride", who);
  if (std::max({p->grad_stride, p->weights ? p->y_stride : 0, p->grad_y_stride}) > INT32_MAX) return fail(LUTKAN_EUNSUPPORTED, "%s: row strides of at most 2^31 - 1", who);
  BackwardArgs a;
  a.grad = static_cast<const unsigned char *>(p->grad); a.y = static_cast<const unsigned char *>(p->y); a.weights = static_cast<const unsigned char *>(p->weights);
  a.rows = p->rows; a.places = p->places; a.grad_y = static_cast<unsigned char *>(p->grad_y); a.grad_weights = static_cast<unsigned char *>(p->grad_weights);
  const int threads = 64 * std::min((p->width + 511) / 512, 16);
  const int64_t check_rows = kCheckRows * threads / 64;
  a.checks = (int32_t)((p->y_rows + check_rows - 1) / check_rows);
  const int64_t groups = p->tokens + a.checks;
  if (groups == 0) return LUTKAN_OK;
  a.y_rows = (int32_t)p->y_rows; a.tokens = (int32_t)p->tokens; a.grad_stride = (int32_t)p->grad_stride; a.y_stride = p->weights ? (int32_t)p->y_stride : 0; a.grad_y_stride = (int32_t)p->grad_y_stride;
  a.top = p->top; a.width = p->width; a.weights_type = (int8_t)p->weights_type; a.rows_bytes = (int8_t)p->rows_bytes; a.places_bytes = (int8_t)p->places_bytes;
  if (!lutkan::launch_holds(groups, threads)) return fail(LUTKAN_EUNSUPPORTED, "%s: too many tokens", who);
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  with_types(p->grad_type, p->y_type, [&](auto g, auto y) { hipLaunchKernelGGL((lutkan_expert_combine_backward_kernel<g, y>), dim3((unsigned)groups), dim3(threads), 0, s, a); });
  return check_launch(who);
}
