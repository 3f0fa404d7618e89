// paged_rows.hip -- writing the paged key/value cache and reading it back (bandwidth-bound).
//
// paged_append_kernel: row r of the n_b new ones of sequence b becomes token L_b - n_b + r, in slot
//   token % page of page table[b][token / page].  8-bit formats: codes and scale of the row by
//   RowScale.
// paged_gather_kernel: the same rows the other way, value = code * scale.
//
// A row (one token, one head) is D channels: D / 8 lanes take 8 each, 16 bytes on the 16-bit side.  A
// workgroup takes 2^tile_shift tokens of one sequence, all heads, K and V.  Its rows run over the tokens
// first, so that neighbouring lane groups touch neighbouring rows of a page.
#include "paged_device.h"

namespace tilemix {

namespace {

constexpr int kRowsThreads = 256;
constexpr int kMaxTileShift = 6;
constexpr int kRowsAhead = 8;   // rows that a lane group has in flight

// Where the tokens of a workgroup lie.
struct RowsTile {
  int first, count;             // packed row of the first token, tokens
  long long token;              // its token number
  __device__ __forceinline__ RowsTile(const PagedRowsArgs& a) {
    const int b = blockIdx.y, t0 = blockIdx.x << a.tile_shift;
    int start, n;
    if (a.cu) {
      start = min(max(a.cu[b], 0), a.total);
      n = min(max(a.cu[b + 1], start), a.total) - start;
    } else {
      start = b * a.len;
      n = a.len;
    }
    first = start + t0;
    count = min(min(n, a.len) - t0, 1 << a.tile_shift);
    token = (long long)a.pool.seqlens[b] - n + t0;
  }
};

// A lane group's row i: token, head and operand.
struct Row {
  int tok, head;
  bool value;
  __device__ __forceinline__ Row(const PagedRowsArgs& a, int i) {
    tok = i & ((1 << a.tile_shift) - 1);
    const int r = i >> a.tile_shift;
    value = r >= a.pool.Hk;
    head = value ? r - a.pool.Hk : r;
  }
};

// Maximum over the D / 8 lanes of a row.
template <int D>
__device__ __forceinline__ uint32_t row_max(uint32_t x) {
  x = max(x, (uint32_t)dpp<0xB1>((int)x, (int)x));
  x = max(x, (uint32_t)dpp<0x4E>((int)x, (int)x));
  x = max(x, (uint32_t)dpp<0x141>((int)x, (int)x));
  if constexpr (D == 128) x = max(x, (uint32_t)dpp<0x140>((int)x, (int)x));
  return x;
}

template <int D, int TYPE, int FORMAT>
__global__ __launch_bounds__(kRowsThreads) void paged_append_kernel(PagedRowsArgs a) {
  constexpr int kLanes = D / 8, kGroups = kRowsThreads / kLanes;
  __shared__ Slot slots[1 << kMaxTileShift];
  const int tid = threadIdx.x, group = tid / kLanes, c = tid % kLanes * 8;
  const RowsTile tile(a);
  if (tile.count <= 0) return;
  if (tid < tile.count) slots[tid] = find_slot(a.pool, blockIdx.y, tile.token + tid);
  __syncthreads();
  const int rows = 2 * a.pool.Hk << a.tile_shift;
  for (int i0 = group; i0 < rows; i0 += kGroups * kRowsAhead) {
    uint4 v[kRowsAhead];
#pragma unroll
    for (int u = 0; u < kRowsAhead; ++u) {
      const Row r(a, i0 + u * kGroups);
      if (i0 + u * kGroups >= rows || r.tok >= tile.count) continue;
      const char* src = static_cast<const char*>(r.value ? a.V : a.K);
      const long long stride = r.value ? a.v_stride : a.k_stride;
      v[u] = ld_global_16(src + 2 * ((tile.first + r.tok) * stride + r.head * D + c));
    }
#pragma unroll
    for (int u = 0; u < kRowsAhead; ++u) {
      const Row r(a, i0 + u * kGroups);
      if (i0 + u * kGroups >= rows || r.tok >= tile.count) continue;   // (alike in a row's lanes)
      const Slot s = slots[r.tok];
      if (s.page < 0) continue;
      const int in_page = (r.head << a.pool.page_shift) + s.slot;
      char* dst = static_cast<char*>(r.value ? a.pool.V : a.pool.K) +
                  kElemBytes<FORMAT> * (s.page * (r.value ? a.pool.stride_v : a.pool.stride_k) + (long long)in_page * D + c);
      if constexpr (!is_8bit(FORMAT)) {
        *reinterpret_cast<uint4*>(dst) = v[u];
      } else {
        const uint32_t w[4] = {v[u].x, v[u].y, v[u].z, v[u].w};
        // Magnitudes compare like their bits; infinities and NaN lie above every finite one.
        u16x2 m = {0, 0};
#pragma unroll
        for (int k = 0; k < 4; ++k) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, w[k] & 0x7fff7fffu));
        const auto s8 = RowScale<FORMAT>::template of<TYPE>(row_max<D>(max((uint32_t)m[0], (uint32_t)m[1])));
        float x[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = bits_to_float<TYPE>(k & 1 ? w[k >> 1] >> 16 : w[k >> 1] & 0xffffu);
        *reinterpret_cast<uint2*>(dst) =
            make_uint2(s8.codes(x[0], x[1], x[2], x[3]), s8.codes(x[4], x[5], x[6], x[7]));
        float* scale = (r.value ? a.pool.dV : a.pool.dK) + s.page * (r.value ? a.pool.stride_dv : a.pool.stride_dk);
        if (c == 0) scale[in_page] = s8.scale;
      }
    }
  }
}

template <int D, int TYPE, int FORMAT>
__global__ __launch_bounds__(kRowsThreads) void paged_gather_kernel(PagedRowsArgs a) {
  constexpr int kLanes = D / 8, kGroups = kRowsThreads / kLanes;
  __shared__ Slot slots[1 << kMaxTileShift];
  const int tid = threadIdx.x, group = tid / kLanes, c = tid % kLanes * 8;
  const RowsTile tile(a);
  if (tile.count <= 0) return;
  if (tid < tile.count) slots[tid] = find_slot(a.pool, blockIdx.y, tile.token + tid);
  __syncthreads();
  const int rows = 2 * a.pool.Hk << a.tile_shift;
  for (int i0 = group; i0 < rows; i0 += kGroups * kRowsAhead) {
    uint4 v[kRowsAhead];
    float scale[kRowsAhead];
#pragma unroll
    for (int u = 0; u < kRowsAhead; ++u) {
      v[u] = make_uint4(0, 0, 0, 0);
      scale[u] = 0.0f;
      const Row r(a, i0 + u * kGroups);
      if (i0 + u * kGroups >= rows || r.tok >= tile.count) continue;
      const Slot s = slots[r.tok];
      if (s.page < 0) continue;
      const int in_page = (r.head << a.pool.page_shift) + s.slot;
      const char* src = static_cast<const char*>(r.value ? a.pool.V : a.pool.K) +
                        kElemBytes<FORMAT> * (s.page * (r.value ? a.pool.stride_v : a.pool.stride_k) + (long long)in_page * D + c);
      if constexpr (!is_8bit(FORMAT)) {
        v[u] = ld_global_16(src);
      } else {
        const uint2 w = *reinterpret_cast<const uint2*>(src);
        v[u].x = w.x;
        v[u].y = w.y;
        scale[u] = ((r.value ? a.pool.dV : a.pool.dK) + s.page * (r.value ? a.pool.stride_dv : a.pool.stride_dk))[in_page];
      }
    }
#pragma unroll
    for (int u = 0; u < kRowsAhead; ++u) {
      const Row r(a, i0 + u * kGroups);
      if (i0 + u * kGroups >= rows || r.tok >= tile.count) continue;
      char* dst = static_cast<char*>(r.value ? a.V : a.K) +
                  2 * ((long long)(tile.first + r.tok) * (r.value ? a.v_stride : a.k_stride) + r.head * D + c);
      if constexpr (is_8bit(FORMAT)) {
        float x[8];
        widen4<FORMAT>(v[u].x, scale[u], *reinterpret_cast<float(*)[4]>(x));
        widen4<FORMAT>(v[u].y, scale[u], *reinterpret_cast<float(*)[4]>(x + 4));
        uint32_t w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = float_to_bits<TYPE>(x[2 * k]) | float_to_bits<TYPE>(x[2 * k + 1]) << 16;
        v[u] = make_uint4(w[0], w[1], w[2], w[3]);
      }
      *reinterpret_cast<uint4*>(dst) = v[u];
    }
  }
}

// Tokens of a workgroup: as many as give each lane group kRowsAhead rows, no more than a sequence can bring.
int tile_shift(const PagedRowsArgs& a, int d) {
  const int groups = kRowsThreads / (d / 8);
  int shift = 0;
  while (shift < kMaxTileShift && (1 << shift) < a.len && (2LL * a.pool.Hk << (shift + 1)) <= (long long)groups * kRowsAhead) ++shift;
  return shift;
}

dim3 rows_grid(const PagedRowsArgs& a) {
  return dim3((unsigned)(((long long)a.len + (1 << a.tile_shift) - 1) >> a.tile_shift), a.pool.B);
}

}  // namespace

hipError_t launch_paged_append(PagedRowsArgs a, int d, int type, int format, hipStream_t stream) {
  a.tile_shift = tile_shift(a, d);
  return for_paged_types(d, type, format, [&](auto D, auto T, auto F) {
    hipLaunchKernelGGL((paged_append_kernel<D(), T(), F()>), rows_grid(a), dim3(kRowsThreads), 0, stream, a);
    return hipGetLastError();
  });
}

hipError_t launch_paged_gather(PagedRowsArgs a, int d, int type, int format, hipStream_t stream) {
  a.tile_shift = tile_shift(a, d);
  return for_paged_types(d, type, format, [&](auto D, auto T, auto F) {
    hipLaunchKernelGGL((paged_gather_kernel<D(), T(), F()>), rows_grid(a), dim3(kRowsThreads), 0, stream, a);
    return hipGetLastError();
  });
}

}  // namespace tilemix
