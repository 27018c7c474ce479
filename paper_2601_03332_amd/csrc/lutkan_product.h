// What the products on 8-bit codes share (lutkan_fp8_matmul.hip, lutkan_int8_matmul.hip): their arguments, rows of codes at any address,
// the search for a tile's group, the place of a piece in LDS, outputs of the three types.
#pragma once

#include "lutkan_fp8.h"

namespace {

// A launch whose arguments take at most 112 bytes costs the host 2.8 us, one with 160 bytes 3.5: lengths and strides travel in 32 bits.
struct ProductArgs {
  const unsigned char *x, *w;
  const float *x_scales, *w_scales;
  unsigned char *y;
  const void *group_sizes, *row_index;
  int64_t w_matrix_stride;
  int32_t x_stride, x_scales_stride, w_stride, y_stride;                             // bytes of codes, elements of scales and outputs
  int32_t rows, x_rows, k, n, groups;
  int8_t y_type, group_sizes_bytes, row_index_bytes;
  int32_t extent;                                                                    // direct: waves of a work-group; tiled: row tiles

  __host__ __device__ int k_blocks() const { return (k + kScaleBlock - 1) / kScaleBlock; }
  __host__ __device__ int n_blocks() const { return (n + kScaleBlock - 1) / kScaleBlock; }
};
static_assert(sizeof(ProductArgs) <= 112, "launch");

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

// Sixteen codes of a row as they are read.  ALIGNED: the row lies at a dword address.  Otherwise the five dwords that hold a byte of
// them (the fifth is the fourth again where the codes lie at one after all), moved into place when they are used, as loads of 16 bytes
// that are not dword-aligned are slower: 70 rows of 4551 -> 240 14.1 -> 8.8 us, 143 of 4395 -> 1504 25 -> 16.
template <bool ALIGNED>
struct Piece {
  u32x4 codes;
  __device__ __forceinline__ void read(const unsigned char *p) { codes = load_any<u32x4>(p); }
  __device__ __forceinline__ u32x4 get(unsigned) const { return codes; }
};
template <>
struct Piece<false> {
  u32x4 first;
  unsigned last;
  __device__ __forceinline__ void read(const unsigned char *p) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(p);
    first = load_any<u32x4>(reinterpret_cast<const unsigned *>(at & ~(uintptr_t)3));
    last = *reinterpret_cast<const unsigned *>((at + 15) & ~(uintptr_t)3);
  }
  // `at`: the low bits of the address they were read from.
  __device__ __forceinline__ u32x4 get(unsigned at) const {
    return u32x4{__builtin_amdgcn_alignbyte(first.y, first.x, at), __builtin_amdgcn_alignbyte(first.z, first.y, at), __builtin_amdgcn_alignbyte(first.w, first.z, at),
                 __builtin_amdgcn_alignbyte(last, first.w, at)};
  }
};

__device__ __forceinline__ unsigned low_bits(const void *p) { return (unsigned)reinterpret_cast<uintptr_t>(p); }

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

// A row's outputs of NT neighbouring column subtiles.  16-bit ones: the 16-lane groups of a pair of subtiles change places, so that a
// lane holds eight neighbouring outputs, 16 bytes, and a store instruction covers 64 bytes of each of its rows instead of 32.
template <int NT>
__device__ __forceinline__ void store_row(const ProductArgs &a, int64_t row, bool exists, int col0, int p, const f32x4 (&v)[NT]) {
  static_assert(NT % 2 == 0, "pairs");
  if (a.y_type == LUTKAN_F32) {
#pragma unroll
    for (int n = 0; n < NT; ++n) if (exists) store_outputs(a, row, col0 + 16 * n + 4 * p, v[n]);
    return;
  }
#pragma unroll
  for (int n = 0; n < NT; n += 2) {
    unsigned bits[2][4];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int e = 0; e < 4; ++e) bits[h][e] = a.y_type == LUTKAN_F16 ? f16_bits(v[n + h][e]) : bf16_bits(v[n + h][e]);
    const u32x2 low = __builtin_amdgcn_permlane16_swap(bits[0][0] | (bits[0][1] << 16), bits[1][0] | (bits[1][1] << 16), false, false);
    const u32x2 high = __builtin_amdgcn_permlane16_swap(bits[0][2] | (bits[0][3] << 16), bits[1][2] | (bits[1][3] << 16), false, false);
    const u32x4 eight{low[0], high[0], low[1], high[1]};
    const int col = col0 + 16 * n + 16 * (p & 1) + 8 * (p >> 1);
    if (!exists || col >= a.n) continue;
    unsigned char *to = a.y + (row * a.y_stride + col) * 2;
    if (col + 8 <= a.n) { store_any(to, eight); continue; }
#pragma unroll
    for (int e = 0; e < 8; ++e) if (col + e < a.n) store_any(to + 2 * e, (unsigned short)(eight[e >> 1] >> ((e & 1) * 16)));
  }
}

// Rows [first, end) of the tile, of one group; group < 0: rows behind the last group, whose outputs are zeros.  end <= first: none.
struct RowTile { int64_t first, end; int group; };

// The sum of v over the lanes up to and with the own one: shifts within rows of 16 lanes, then the rows' ends handed on.
__device__ __forceinline__ int lanes_below(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, true);       // row_shr:1
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, true);       // lane 15 of a row to the next, in rows 1 and 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, true);       // lane 31 to rows 2 and 3
  return v;
}

// 64 groups, a lane each: the rows of a group and its tiles of HEIGHT rows, counted from the first group on.  The sizes are the caller's,
// on the device: negative ones count as none, and a group ends with the rows at the latest.  (At most 2^24 rows: sums of 64 sizes
// stay below 2^31.)
template <int HEIGHT>
struct GroupTiles {
  int first, end, tiles_before, tiles_with;
  __device__ __forceinline__ GroupTiles(const ProductArgs &a, int base, int row0, int tile0) {
    const int group = base + (threadIdx.x & 63), rows = a.rows;
    int size = 0;
    if (group < a.groups) {
      if (a.group_sizes_bytes == 8) size = (int)max((int64_t)0, min(static_cast<const int64_t *>(a.group_sizes)[group], (int64_t)rows));
      else size = max(0, min(static_cast<const int32_t *>(a.group_sizes)[group], rows));
    }
    const int with = lanes_below(size);
    first = min(row0 + with - size, rows);
    end = min(row0 + with, rows);
    const int own = (end - first + HEIGHT - 1) / HEIGHT;
    tiles_with = tile0 + lanes_below(own);
    tiles_before = tiles_with - own;
  }
};

// A tile of the rows, cut at the groups' ends: every group's rows in tiles of HEIGHT, then those behind the last group.  Each wave for
// itself.  tile_of(number of all tiles): which one, negative: none.
template <int HEIGHT, typename TileOf>
__device__ __forceinline__ RowTile grouped_tile(const ProductArgs &a, const TileOf &tile_of) {
  int row = 0, tiles = 0, base = 0;
  GroupTiles<HEIGHT> g(a, 0, 0, 0);
  for (;;) {                                                     // all tiles
    row = __builtin_amdgcn_readlane(g.end, 63);
    tiles = __builtin_amdgcn_readlane(g.tiles_with, 63);
    if (base + 64 >= a.groups) break;
    base += 64;
    g = GroupTiles<HEIGHT>(a, base, row, tiles);
  }
  const int rows = a.rows, behind = row, first_behind = tiles;
  const int tile = tile_of(tiles + (rows - row + HEIGHT - 1) / HEIGHT);
  if (tile < 0) return {0, 0, 0};
  if (tile >= first_behind) {
    const int at = behind + (tile - first_behind) * HEIGHT;
    return {at, min(at + HEIGHT, rows), -1};
  }
  if (base > 0) g = GroupTiles<HEIGHT>(a, base = 0, 0, 0);
  for (;;) {
    const unsigned long long here = __ballot(tile < g.tiles_with);
    if (here != 0) {
      const int owner = __builtin_ctzll(here);
      const int at = __builtin_amdgcn_readlane(g.first, owner) + (tile - __builtin_amdgcn_readlane(g.tiles_before, owner)) * HEIGHT;
      return {at, min(at + HEIGHT, __builtin_amdgcn_readlane(g.end, owner)), base + owner};
    }
    base += 64;                                                  // (tile < first_behind: some group has it)
    g = GroupTiles<HEIGHT>(a, base, __builtin_amdgcn_readlane(g.end, 63), __builtin_amdgcn_readlane(g.tiles_with, 63));
  }
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

// The 16-byte piece `piece` of a row's eight lies in LDS at this place of them (its own inverse).
__device__ __forceinline__ int piece_place(int row, int piece) { return piece ^ ((row >> 1) & 7); }

// As copy16_global_to_lds_at, four bytes a lane.
__device__ __forceinline__ void copy4_global_to_lds_at(const void *uniform_base, unsigned lane_byte_offset, void *lds_dst) {
  const unsigned dst = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)(__attribute__((address_space(3))) void *)lds_dst);
  if constexpr (kLdsDmaPreservesM0) {
    unsigned saved;
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %2, %3\n\ts_mov_b32 m0, %0"
                 : "=&s"(saved) : "s"(dst), "v"(lane_byte_offset), "s"(uniform_base) : "memory");
  } else {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(dst), "v"(lane_byte_offset), "s"(uniform_base) : "m0", "memory");
  }
}

bool rows_aligned(const ProductArgs &a) {                        // every row at a dword address
  return ((reinterpret_cast<uintptr_t>(a.x) | reinterpret_cast<uintptr_t>(a.w) | (uintptr_t)a.x_stride | (uintptr_t)a.w_stride | (uintptr_t)a.w_matrix_stride) & 3) == 0;
}
template <bool GROUPED>
bool copies_fit(const ProductArgs &a) {                          // the rows' offsets, as the copies hold them
  const int64_t x_span = GROUPED ? std::max(a.x_rows, 1) : 256, most = ((int64_t)1 << 32) - kScaleBlock;     // (a block's columns beside them)
  return a.x_stride < most / x_span && a.x_scales_stride < most / 4 / x_span && a.w_stride < most / 256;
}

}  // namespace
