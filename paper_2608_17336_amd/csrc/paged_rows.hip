// paged_rows.hip -- writing the paged key/value cache and reading it back (bandwidth-bound).
//
// paged_append_kernel: row r of the n_b new ones of sequence b becomes token L_b - n_b + r, in slot
//   token % page of page table[b][token / page].  8-bit formats: codes and scale of the row by
//   RowScale; MXFP4: codes and exponents of its blocks by block_exponent and codes8.
// paged_gather_kernel: the same rows the other way, value = code * scale.
//
// A row (one token, one head) is D channels: D / 8 lanes take 8 each, 16 bytes on the 16-bit side.  A
// workgroup takes 2^tile_shift tokens of one sequence and all heads of K and V, which is one run of the 16-bit
// side, where most of the bytes are; a lane group takes one token of them and some of its heads, so that it
// finds the token's slot once and steps through the heads by additions.  (32 tokens and few heads, whole cache
// lines of an 8-bit cache and its scales, were 8% slower: 24 prompts of up to 16000 tokens, E4M3, 8 heads of d = 128,
// 97 us to append where this shape took 84.)
#include "paged_device.h"

#include <algorithm>

namespace tilemix {

namespace {

constexpr int kRowsThreads = 256;
// Rows that a lane group requests at a time: few, so that many waves fit and their requests overlap.  us to append
// (24 prompts of up to 16000 tokens, E4M3, 8 heads of d = 128) and read back, with the same rows of a group in
// all: 8 at a time 140.1, 4 133.5, 2 131.1.
constexpr int kRowsAhead = 2;
// Rows that a lane group takes in all, at most.  us, of the same and of reading 12 prefixes of up to 32768
// tokens (INT8): appended 2 rows and read 4 116.2 and 94.2, 4 and 4 111.0 and 94.2, 4 and 8 111.2 and 99.1, 8 and 4 112.7 and
// 93.9, 4 and 2 119.3 and 111.8.  Read out of MXFP4 at d = 128, whose rows are 64 bytes, with 4 and with 8: 8 heads 96.8 and 96.8,
// 16 55.8 and 52.2, 32 136 and 131 (d = 64: 8 heads 35.8 and 37.1, 32 110 and 112).
constexpr int kRows = 4;
constexpr int gather_rows(int d, int format) { return is_4bit(format) && d == 128 ? 2 * kRows : kRows; }
// Adjacent tiles for one XCD: workgroups are dealt to the 8 XCDs in turn, and a tile's scales and exponents are parts of
// cache lines, which are moved once where one L2 has all parts.  us, as before, in MXFP4: 1 tile 98.5 and 97.6, 4 96.8 and 97.5, 8 96.0
// and 97.0, 32 95.1 and 96.8, 128 95.3 and 97.5, 512 97.9 and 100.4; in E4M3 and INT8 1 112.5 and 99.2, 32 111.2 and 99.1.
constexpr int kXcdTiles = 32;

// The tokens of a workgroup.  Those of a packed batch are numbered in tiles, sequence after sequence, which
// every wave looks up for itself (a lane takes a run of sequences): a grid over the longest sequence would be
// mostly empty for lengths that differ.
struct RowsTile {
  int b = 0, first = 0, count = 0;   // sequence, packed row of the first token, tokens
  long long token = 0;               // its token number
  __device__ __forceinline__ RowsTile(const PagedRowsArgs& a, int lane) {
    const int size = 1 << a.tile_shift, i = blockIdx.x % (8 * kXcdTiles), first_of = blockIdx.x - i;   // i-th of 8 kXcdTiles
    // (Behind the last 8 kXcdTiles they stay in order.)
    const int id = first_of + (first_of + 8 * kXcdTiles <= (int)gridDim.x ? i % 8 * kXcdTiles + i / 8 : i);
    int start, n, t0;
    if (a.cu) {
      const int B = a.pool.B, per = (B + kWave - 1) / kWave, b0 = min(lane * per, B), b1 = min(b0 + per, B);
      auto rows = [&](int s, int& from) {
        from = min(max(a.cu[s], 0), a.total);
        return min(max(a.cu[s + 1], from), a.total) - from;
      };
      auto tiles = [&](int rows) { return (min(rows, a.len) + size - 1) >> a.tile_shift; };
      int own = 0, from = 0, mine = 0;
      for (int s = b0; s < b1; ++s) {
        mine = rows(s, from);
        own += tiles(mine);
      }
      const int end = wave_scan(own);
      int at = end - own, seq = b0, tile = 0;
      const bool hit = id >= at && id < end;
      const uint64_t hits = __ballot(hit);
      if (!hits) return;
      if (hit) {
        for (int s = b0; s < b1; ++s) {
          if (per > 1) mine = rows(s, from);   // (a single one is at hand)
          const int k = tiles(mine);
          if (id < at + k) {
            seq = s;
            tile = id - at;
            break;
          }
          at += k;
        }
      }
      const int l = __builtin_ctzll(hits);
      b = __builtin_amdgcn_readlane(seq, l);
      start = __builtin_amdgcn_readlane(from, l);
      n = __builtin_amdgcn_readlane(mine, l);
      t0 = __builtin_amdgcn_readlane(tile, l) << a.tile_shift;
    } else {
      b = (int)a.div_tiles.quot(id);
      start = b * a.len;
      n = a.len;
      t0 = (id - b * (int)a.div_tiles.d) << a.tile_shift;
    }
    first = start + t0;
    count = min(min(n, a.len) - t0, size);
    token = (long long)a.pool.seqlens[b] - n + t0;
  }
};

// What a lane group does: token tok of the tile, and of the token's 2 Hk rows (K's heads, then V's) row r0 and every
// step-th one after it.
struct LaneGroup {
  int tok, r0, step;
  __device__ __forceinline__ LaneGroup(const PagedRowsArgs& a, int group, int groups)
      : tok(group & ((1 << a.tile_shift) - 1)), r0(group >> a.tile_shift), step(groups >> a.tile_shift) {}
};

// Where a token's rows lie in a tensor pair: K's head h at K + h step bytes, V's alike.
struct RowPointers {
  char *K, *V;
  long long step;
  __device__ __forceinline__ char* row(int r, int Hk) const { return r < Hk ? K + r * step : V + (r - Hk) * step; }
};

template <int D>
__device__ __forceinline__ RowPointers packed_rows(const PagedRowsArgs& a, long long row, int c) {
  return {static_cast<char*>(a.K) + 2 * (row * a.k_stride + c), static_cast<char*>(a.V) + 2 * (row * a.v_stride + c), 2 * D};
}

template <int D, int FORMAT>
__device__ __forceinline__ RowPointers cached_rows(const PagedPool& p, const Slot& s, int c) {
  constexpr int kRow = kRowBytes<D, FORMAT>;
  const long long in = (long long)s.slot * kRow + c * kRow / D;
  return {static_cast<char*>(p.K) + s.page * p.stride_k * kElemBytes<FORMAT> + in,
          static_cast<char*>(p.V) + s.page * p.stride_v * kElemBytes<FORMAT> + in, (long long)kRow << p.page_shift};
}

// The row's scale, or the exponent of the channel's block.
template <int D, int FORMAT>
__device__ __forceinline__ RowPointers cached_scales(const PagedPool& p, const Slot& s, int c) {
  constexpr int kRow = kScaleBytes<D, FORMAT>, kElem = is_4bit(FORMAT) ? 1 : 4;
  const long long in = (long long)s.slot * kRow + (is_4bit(FORMAT) ? c / 32 : 0);
  return {static_cast<char*>(p.dK) + s.page * p.stride_dk * kElem + in,
          static_cast<char*>(p.dV) + s.page * p.stride_dv * kElem + in, (long long)kRow << p.page_shift};
}

// Maximum over the LANES lanes of a row or block.
template <int LANES>
__device__ __forceinline__ uint32_t lanes_max(uint32_t x) {
  x = max(x, (uint32_t)dpp<0xB1>((int)x, (int)x));
  x = max(x, (uint32_t)dpp<0x4E>((int)x, (int)x));
  if constexpr (LANES >= 8) x = max(x, (uint32_t)dpp<0x141>((int)x, (int)x));
  if constexpr (LANES >= 16) x = max(x, (uint32_t)dpp<0x140>((int)x, (int)x));
  return x;
}

template <int D, int TYPE, int FORMAT>
__global__ __launch_bounds__(kRowsThreads) void paged_append_kernel(PagedRowsArgs a) {
  constexpr int kLanes = D / 8, kGroups = kRowsThreads / kLanes;
  const int tid = threadIdx.x, c = tid % kLanes * 8, Hk = a.pool.Hk, rows = 2 * Hk;
  const RowsTile tile(a, tid & (kWave - 1));
  const LaneGroup g(a, tid / kLanes, kGroups);
  if (g.tok >= tile.count) return;   // (alike in a row's lanes, as all that follows)
  const RowPointers src = packed_rows<D>(a, tile.first + g.tok, c);
  uint4 v[kRowsAhead];
  auto load = [&](int r0) {
#pragma unroll
    for (int u = 0; u < kRowsAhead; ++u)
      if (r0 + u * g.step < rows) v[u] = ld_global_16(src.row(r0 + u * g.step, Hk));
  };
  load(g.r0);   // before the slot is looked up
  const Slot s = find_slot(a.pool, tile.b, tile.token + g.tok);
  if (s.page < 0) return;
  const RowPointers dst = cached_rows<D, FORMAT>(a.pool, s, c), scales = cached_scales<D, FORMAT>(a.pool, s, c);
  for (int r0 = g.r0; r0 < rows; r0 += g.step * kRowsAhead) {
    if (r0 != g.r0) load(r0);
#pragma unroll
    for (int u = 0; u < kRowsAhead; ++u) {
      const int r = r0 + u * g.step;
      if (r >= rows) break;
      if constexpr (!is_8bit(FORMAT) && !is_4bit(FORMAT)) {
        *reinterpret_cast<uint4*>(dst.row(r, Hk)) = v[u];
      } else {
        const uint32_t w[4] = {v[u].x, v[u].y, v[u].z, v[u].w};
        // Magnitudes compare like their bits; infinities and NaN lie above every finite one.
        u16x2 m = {0, 0};
#pragma unroll
        for (int k = 0; k < 4; ++k) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, w[k] & 0x7fff7fffu));
        const uint32_t own = max((uint32_t)m[0], (uint32_t)m[1]);
        if constexpr (is_4bit(FORMAT)) {
          const uint32_t e = block_exponent<TYPE>(lanes_max<4>(own));
          *reinterpret_cast<uint32_t*>(dst.row(r, Hk)) = codes8<TYPE>(w, e);
          if (c % 32 == 0) *reinterpret_cast<uint8_t*>(scales.row(r, Hk)) = (uint8_t)e;
        } else {
          const auto s8 = RowScale<FORMAT>::template of<TYPE>(lanes_max<kLanes>(own));
          float x[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) x[k] = bits_to_float<TYPE>(k & 1 ? w[k >> 1] >> 16 : w[k >> 1] & 0xffffu);
          *reinterpret_cast<uint2*>(dst.row(r, Hk)) =
              make_uint2(s8.codes(x[0], x[1], x[2], x[3]), s8.codes(x[4], x[5], x[6], x[7]));
          if (c == 0) *reinterpret_cast<float*>(scales.row(r, Hk)) = s8.scale;
        }
      }
    }
  }
}

// Rows of this many bytes and more are written past the caches, which then keep the pool.  us, 12 prefixes out of an MXFP4
// pool: 73 MB of rows 19.0, so 16.2; 204 MB 64.9 and 40.9; 361 MB 110.5 and 96.8 (out of INT8 102.1 and 94.1); 24 prompts
// appended to MXFP4 and read back, 201 MB, 126.4 and 94.7.  But their reader finds less in the caches: with a prefill of 16
// tokens a sequence over them 113 MB 124 and 129, 148 MB 160 and 165, 183 MB 210 and 207, 226 MB 260 and 258, 355 MB 458 and 438.
constexpr long long kStreamBytes = 160 << 20;

template <int D, int TYPE, int FORMAT, bool STREAM>
__global__ __launch_bounds__(kRowsThreads) void paged_gather_kernel(PagedRowsArgs a) {
  constexpr int kLanes = D / 8, kGroups = kRowsThreads / kLanes;
  const int tid = threadIdx.x, c = tid % kLanes * 8, Hk = a.pool.Hk, rows = 2 * Hk;
  const RowsTile tile(a, tid & (kWave - 1));
  const LaneGroup g(a, tid / kLanes, kGroups);
  if (g.tok >= tile.count) return;
  const RowPointers dst = packed_rows<D>(a, tile.first + g.tok, c);
  Slot s = find_slot(a.pool, tile.b, tile.token + g.tok);
  const bool some = s.page >= 0;
  s.page = max(s.page, 0);   // nothing is read where there is no page
  const RowPointers src = cached_rows<D, FORMAT>(a.pool, s, c), scales = cached_scales<D, FORMAT>(a.pool, s, c);
  for (int r0 = g.r0; r0 < rows; r0 += g.step * kRowsAhead) {
    uint4 v[kRowsAhead];
    float scale[kRowsAhead];
#pragma unroll
    for (int u = 0; u < kRowsAhead; ++u) {
      const int r = r0 + u * g.step;
      v[u] = make_uint4(0, 0, 0, 0);
      scale[u] = 0.0f;
      if (r >= rows || !some) continue;
      if constexpr (is_4bit(FORMAT)) {
        v[u].x = *reinterpret_cast<const uint32_t*>(src.row(r, Hk));
        scale[u] = block_scale(*reinterpret_cast<const uint8_t*>(scales.row(r, Hk)));
      } else if constexpr (!is_8bit(FORMAT)) {
        v[u] = ld_global_16(src.row(r, Hk));
      } else {
        const uint2 w = *reinterpret_cast<const uint2*>(src.row(r, Hk));
        v[u].x = w.x;
        v[u].y = w.y;
        scale[u] = *reinterpret_cast<const float*>(scales.row(r, Hk));
      }
    }
#pragma unroll
    for (int u = 0; u < kRowsAhead; ++u) {
      const int r = r0 + u * g.step;
      if (r >= rows) break;
      if constexpr (is_4bit(FORMAT)) {
        v[u] = mx_values8<TYPE>(v[u].x, scale[u]);
      } else if constexpr (is_8bit(FORMAT)) {
        float x[8];
        widen4<FORMAT>(v[u].x, scale[u], *reinterpret_cast<float(*)[4]>(x));
        widen4<FORMAT>(v[u].y, scale[u], *reinterpret_cast<float(*)[4]>(x + 4));
        uint32_t w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = float_to_bits<TYPE>(x[2 * k]) | float_to_bits<TYPE>(x[2 * k + 1]) << 16;
        v[u] = make_uint4(w[0], w[1], w[2], w[3]);
      }
      typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
      u32x4* to = reinterpret_cast<u32x4*>(dst.row(r, Hk));
      if constexpr (STREAM) __builtin_nontemporal_store(__builtin_bit_cast(u32x4, v[u]), to);
      else *to = __builtin_bit_cast(u32x4, v[u]);
    }
  }
}

// Tokens of a workgroup: the most, no more than lane groups and than a sequence can bring, with which a lane group has
// at most `most` rows.
dim3 rows_grid(PagedRowsArgs& a, int d, int most) {
  const int groups = kRowsThreads / (d / 8);
  a.tile_shift = 0;
  while ((2 << a.tile_shift) <= groups && (1 << a.tile_shift) < a.len &&
         (2LL * a.pool.Hk << (a.tile_shift + 1)) <= (long long)groups * most)
    ++a.tile_shift;
  const long long per = ((long long)a.len + (1 << a.tile_shift) - 1) >> a.tile_shift;   // tiles of the longest sequence
  a.div_tiles = FastDiv((uint32_t)per);
  long long tiles = per * a.pool.B;
  if (a.cu) tiles = std::min(tiles, ((long long)a.total >> a.tile_shift) + a.pool.B);
  return dim3((unsigned)tiles);
}

}  // namespace

hipError_t launch_paged_append(PagedRowsArgs a, int d, int type, int format, hipStream_t stream) {
  const dim3 grid = rows_grid(a, d, kRows);
  return for_paged_types(d, type, format, [&](auto D, auto T, auto F) {
    hipLaunchKernelGGL((paged_append_kernel<D(), T(), F()>), grid, dim3(kRowsThreads), 0, stream, a);
    return hipGetLastError();
  });
}

hipError_t launch_paged_gather(PagedRowsArgs a, int d, int type, int format, hipStream_t stream) {
  const dim3 grid = rows_grid(a, d, gather_rows(d, format));
  return for_paged_types(d, type, format, [&](auto D, auto T, auto F) {
    if (4LL * a.total * a.pool.Hk * d >= kStreamBytes)
      hipLaunchKernelGGL((paged_gather_kernel<D(), T(), F(), true>), grid, dim3(kRowsThreads), 0, stream, a);
    else
      hipLaunchKernelGGL((paged_gather_kernel<D(), T(), F(), false>), grid, dim3(kRowsThreads), 0, stream, a);
    return hipGetLastError();
  });
}

}  // namespace tilemix
