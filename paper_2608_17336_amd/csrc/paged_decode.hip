// paged_decode.hip -- one decode step over the paged key/value cache.
//
// For query head hq of sequence b, over the tokens j attended to (the last `window`, or all, whose page
// exists): s_j = scale q . k_j, O = sum_j e^(s_j - m) v_j / sum_j e^(s_j - m), lse = m + ln of that sum.
//
//   paged_decode_kernel: workgroup (chunk of tiles, KV head and block of 16 query heads, sequence), 4 waves.
//     Each wave streams tiles of the chunk with a running (max, normalizer, output) of its own in
//     registers; they are joined in LDS, and the workgroup writes O, or the chunk's partial result
//     where the sequence has several chunks.
//   paged_join_kernel: joins the chunks of one (sequence, query head) by their log-sum-exp.
//
// Bound: HBM.  Each cached row is read once per block of 16 query heads, with O(1) work per byte.
#include "paged_device.h"

#include <algorithm>

namespace tilemix {

namespace {

constexpr int kPagedWaves = 4;
constexpr int kPagedHeads = 16;                  // query heads on the columns of a matrix-core tile
// Workgroups that share the tiles of a batch.
constexpr int kPagedWorkgroups = 768;

// 16-key slabs per tile: a tile is 16 KiB of K and V for d = 128, 8 KiB for d = 64.
template <int FORMAT>
constexpr int kSlabs = is_8bit(FORMAT) ? 4 : 2;

int tile_keys(int format) { return 16 * (format == TILEMIX_INT8 || format == TILEMIX_E4M3 ? 4 : 2); }

// The tokens that a sequence's query attends to, as tiles of `keys` tokens: first .. len - 1, of tiles
// first / keys .. .
struct Span {
  int first, len, tile0, tiles;
  __device__ __forceinline__ Span(const PagedDecodeArgs& a, int b, int keys) {
    const PagedPool& p = a.pool;
    len = min(max(p.seqlens[b], 0), p.max_pages << p.page_shift);
    first = a.window > 0 ? max(len - a.window, 0) : 0;
    tile0 = first / keys;
    tiles = (len + keys - 1) / keys - tile0;
  }
};

// How the batch is cut: every sequence into chunks of `tiles` tiles (the last one maybe fewer; one empty
// chunk where it has no token), the fewest tiles, the same number for every wave, with which the chunks of
// all heads fit the workgroups.  Found by every wave for itself: a lane takes a run of sequences.
struct Chunk {
  int b = -1, index, count, tiles;   // b = -1: no chunk for this workgroup
  int head_block;                    // KV head and block of query heads
  int first_id;                      // workgroup of the sequence's and head block's chunk 0
  __device__ __forceinline__ Chunk(const PagedDecodeArgs& a, int id, int lane, int keys) {
    const int B = a.pool.B, per = (B + kWave - 1) / kWave, b0 = lane * per, b1 = min(b0 + per, B);
    int sum = 0;
    for (int s = b0; s < b1; ++s) sum += Span(a, s, keys).tiles;
    const int total = __builtin_amdgcn_readlane(wave_scan(sum), kWave - 1);
    const int share = a.chunk_workgroups * kPagedWaves;
    tiles = kPagedWaves * max(1, (int)(((long long)total * a.head_blocks + share - 1) / share));
    int mine = 0;
    for (int s = b0; s < b1; ++s) mine += max(1, (Span(a, s, keys).tiles + tiles - 1) / tiles);
    const int end = wave_scan(mine), all = __builtin_amdgcn_readlane(end, kWave - 1);
    head_block = id / all;
    if (head_block >= a.head_blocks) return;
    const int slot = id - head_block * all;
    int at = end - mine, seq = 0, idx = 0, cnt = 0;
    const bool hit = slot >= at && slot < end;
    if (hit) {
      for (int s = b0; s < b1; ++s) {
        const int n = max(1, (Span(a, s, keys).tiles + tiles - 1) / tiles);
        if (slot < at + n) {
          seq = s;
          idx = slot - at;
          cnt = n;
          break;
        }
        at += n;
      }
    }
    const int l = __builtin_ctzll(__ballot(hit));
    b = __builtin_amdgcn_readlane(seq, l);
    index = __builtin_amdgcn_readlane(idx, l);
    count = __builtin_amdgcn_readlane(cnt, l);
    first_id = id - index;
  }
};

// Matrix-core products with 16-bit operands as the cache needs them: BF16 for a BF16 cache, else FP16 (8-bit
// codes are exact in FP16).
template <int FORMAT>
__device__ __forceinline__ f32x4 mfma_16(uint4 x, uint4 y, f32x4 c) {
  if constexpr (FORMAT == TILEMIX_BF16)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(as_half8(x), as_half8(y), c, 0, 0, 0);
}

typedef _Float16 half2_t __attribute__((ext_vector_type(2)));

// Codes 2 w, 2 w + 1 of four E4M3 codes, in FP16.
template <bool HIGH>
__device__ __forceinline__ uint32_t e4m3x2_to_half2(uint32_t w) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w, 1.0f, HIGH));
}

// Eight codes in FP16.
template <int FORMAT>
__device__ __forceinline__ uint4 widen8(uint32_t w0, uint32_t w1) {
  if constexpr (FORMAT == TILEMIX_INT8)
    return __builtin_bit_cast(uint4, i8x8_to_half8(w0, w1));
  else
    return make_uint4(e4m3x2_to_half2<false>(w0), e4m3x2_to_half2<true>(w0), e4m3x2_to_half2<false>(w1),
                      e4m3x2_to_half2<true>(w1));
}

__device__ __forceinline__ float quad_rows_sum(float x) {
  const int v = __builtin_bit_cast(int, x);
  const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  return pair_sum(__builtin_bit_cast(float, (int)r[0]) + __builtin_bit_cast(float, (int)r[1]));
}

// Weights are formed as 2^(s - m + kShift) so that their FP16 pieces reach far below the largest:
// two pieces hold a weight to 2^-22 of itself down to 2^-29 of the largest and to 2^-40 of it below.  BF16
// pieces have FP32's range.
template <int FORMAT>
constexpr float kShift = FORMAT == TILEMIX_BF16 ? 0.0f : 15.0f;

// Two 16-bit pieces of four weights.
template <int FORMAT>
__device__ __forceinline__ void split4(const float (&w)[4], uint2& hi, uint2& lo) {
  constexpr int kMath = FORMAT == TILEMIX_BF16 ? TILEMIX_BF16 : TILEMIX_FP16;
  uint32_t h[4], l[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    h[r] = float_to_bits<kMath>(w[r]);
    l[r] = float_to_bits<kMath>(w[r] - bits_to_float<kMath>(h[r]));
  }
  hi = make_uint2(h[0] | h[1] << 16, h[2] | h[3] << 16);
  lo = make_uint2(l[0] | l[1] << 16, l[2] | l[3] << 16);
}

// Scores are computed transposed, S^T = K Q^T: a slab's 16 keys on the rows, the query heads on the columns
// of a 16x16 product, so that lane (l16, lq) = (lane % 16, lane / 16) receives keys 4 lq + r (r < 4) of
// head l16.  For the pair of slabs 2 t, 2 t + 1 these are the eight keys that the B operand of
// O^T += V^T P^T wants in that lane, so P stays in registers.  The A operand V^T wants the same keys of
// channel row l16; row i of product c is given channel i D / 16 + c, so that a lane reads D / 16
// adjacent channels of a key at once and pairs the keys by byte permutes: no transposed copy of V is
// kept, and a row can be appended to a page as it is.
template <int D, int TYPE, int FORMAT>
__global__ __launch_bounds__(kPagedWaves * kWave) __attribute__((amdgpu_waves_per_eu(2)))
void paged_decode_kernel(PagedDecodeArgs a) {
  constexpr int kS = kSlabs<FORMAT>, kKeys = 16 * kS;
  constexpr int kBytes = kElemBytes<FORMAT>;
  constexpr bool k8 = is_8bit(FORMAT);
  constexpr int kKL = D * kBytes / 64;             // 16-byte loads of a key row per lane
  constexpr int kC = D / 16;                       // channels of a lane's value row: output products
  constexpr int kVW = kC * kBytes / 4;             // dwords of them
  constexpr int kQ = D / 32;                       // score products per slab
  constexpr int kOS = D + 4;                       // padded LDS row
  const PagedPool& p = a.pool;
  const int tid = threadIdx.x, lane = tid & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int l16 = lane & 15, lq = lane >> 4;
  const float ninf = -__builtin_huge_valf();
  const Chunk ch(a, blockIdx.x, lane, kKeys);
  if (ch.b < 0) return;
  const int b = ch.b, G = a.Hq / p.Hk, blocks = a.head_blocks / p.Hk;
  const int hk = ch.head_block / blocks, g0 = ch.head_block % blocks * kPagedHeads;
  const int heads = min(kPagedHeads, G - g0), hq0 = hk * G + g0;
  const Span span(a, b, kKeys);
  const int tile0 = span.tile0 + ch.index * ch.tiles;
  const int tile_end = min(tile0 + ch.tiles, span.tile0 + span.tiles);

  __shared__ float red_m[kPagedWaves][kPagedHeads], red_z[kPagedWaves][kPagedHeads];
  __shared__ int red_e[kPagedWaves];
  __shared__ __align__(16) float osum[kPagedWaves][kPagedHeads][kOS];

  // 1. Page ids of the wave's tiles tile0 + wave + i kPagedWaves, 64 at a time: lane (i, j) holds the j-th of
  //    the 2^per_shift pages of tile i.
  const int keys_shift = 4 + (kS == 8 ? 3 : kS == 4 ? 2 : 1);
  const int per_shift = max(0, keys_shift - p.page_shift);
  const int* table = p.table + b * p.stride_table;
  auto load_ids = [&](int i0) {
    const int i = i0 + (lane >> per_shift), n = tile0 + wave + i * kPagedWaves;
    const long long e = ((long long)n * kKeys >> p.page_shift) + (lane & ((1 << per_shift) - 1));
    int id = -1;
    if (n < tile_end && e < p.max_pages && (e << p.page_shift) < span.len) id = table[e];
    return id >= 0 && id < p.pages ? id : -1;
  };
  int ids = load_ids(0);
  const int id_tiles = kWave >> per_shift;

  // 2. One tile in registers.
  uint4 kr[kS][kKL];
  uint32_t vr[kS][4][kVW];
  f32x4 dk[kS], dv[kS];
  int page[kS];                                    // of the tile that is requested next, per slab
  const char* poolK = static_cast<const char*>(p.K);
  const char* poolV = static_cast<const char*>(p.V);
  const uint32_t k_off = (uint32_t)(l16 * D * kBytes + 16 * lq);
  const uint32_t v_off = (uint32_t)(4 * lq * D * kBytes + l16 * kC * kBytes);
  auto find_pages = [&](int i) {
    const int at = (i & (id_tiles - 1)) << per_shift;
#pragma unroll
    for (int s = 0; s < kS; ++s) page[s] = __builtin_amdgcn_readlane(ids, at + (16 * s >> p.page_shift));
  };
  // Rows of slab s of tile n in page `id`, or of page 0 where there is none: they are masked.
  auto slab_row = [&](int n, int s) { return (hk << p.page_shift) + ((n * kKeys + 16 * s) & ((1 << p.page_shift) - 1)); };
  auto load_keys = [&](int n) {
#pragma unroll
    for (int s = 0; s < kS; ++s) {
      const char* base = poolK + kBytes * (max(page[s], 0) * p.stride_k + (long long)slab_row(n, s) * D);
#pragma unroll
      for (int i = 0; i < kKL; ++i) kr[s][i] = ld_global_16(base + 64 * i + k_off);
    }
  };
  auto load_values = [&](int n) {
#pragma unroll
    for (int s = 0; s < kS; ++s) {
      const char* base = poolV + kBytes * (max(page[s], 0) * p.stride_v + (long long)slab_row(n, s) * D);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const char* at = base + r * D * kBytes + v_off;
        if constexpr (kVW == 4) {
          const uint4 x = ld_global_16(at);
          vr[s][r][0] = x.x; vr[s][r][1] = x.y; vr[s][r][2] = x.z; vr[s][r][3] = x.w;
        } else if constexpr (kVW == 2) {
          const uint2 x = *reinterpret_cast<const uint2*>(at);
          vr[s][r][0] = x.x; vr[s][r][1] = x.y;
        } else {
          vr[s][r][0] = *reinterpret_cast<const uint32_t*>(at);
        }
      }
    }
  };
  auto load_scales = [&](int n) {
    if constexpr (k8) {
#pragma unroll
      for (int s = 0; s < kS; ++s) {
        const int row = slab_row(n, s) + 4 * lq;
        dk[s] = *reinterpret_cast<const f32x4*>(p.dK + max(page[s], 0) * p.stride_dk + row);
        dv[s] = *reinterpret_cast<const f32x4*>(p.dV + max(page[s], 0) * p.stride_dv + row);
      }
    }
  };

  // 3. Query rows as the B operand of the score products: lane (head l16, lq) holds the channels that it
  //    reads of a key row.  BF16 queries against 8-bit codes are brought to FP16 by a power of two per
  //    head, 2^q_exp: the largest to [2^14, 2^15), so that what FP16 cannot hold lies below 2^-39 of it.
  uint4 qf[kQ];
  int q_exp = 0;
  {
    const char* q = static_cast<const char*>(a.Q) + 2 * (b * a.q_stride + (long long)(hq0 + min(l16, heads - 1)) * D);
#pragma unroll
    for (int i = 0; i < kQ; ++i) {
      const int c = k8 ? 64 * (i / 2) + 16 * lq + 8 * (i % 2) : 32 * i + 8 * lq;
      qf[i] = ld_global_16(q + 2 * c);
      if (l16 >= heads) qf[i] = make_uint4(0, 0, 0, 0);
    }
    if constexpr (k8 && TYPE == TILEMIX_BF16) {
      float x[kQ][8], amax = 0.0f;
#pragma unroll
      for (int i = 0; i < kQ; ++i) {
        const uint32_t w[4] = {qf[i].x, qf[i].y, qf[i].z, qf[i].w};
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          x[i][e] = bits_to_float<TILEMIX_BF16>(e & 1 ? w[e >> 1] >> 16 : w[e >> 1] & 0xffffu);
          amax = fmaxf(amax, fabsf(x[i][e]));
        }
      }
      q_exp = 15 - __builtin_amdgcn_frexp_expf(quad_rows_max(amax));
#pragma unroll
      for (int i = 0; i < kQ; ++i) {
        uint32_t w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = float_to_bits<TILEMIX_FP16>(__builtin_amdgcn_ldexpf(x[i][e], q_exp));
        qf[i] = make_uint4(w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16, w[6] | w[7] << 16);
      }
    }
  }

  // 4. The wave's tiles.  m, z: running max (log2 units) and this lane's share of the normalizer; acc: output in
  //    units of 2^e.  e follows the largest value scale so far, so that p dV, the weight of a code, fits
  //    FP16 pieces whatever the values' size.
  float m = ninf, z = 0.0f;
  int e = -2048;
  f32x4 acc[kC];
#pragma unroll
  for (int c = 0; c < kC; ++c) acc[c] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  int i = 0, n = tile0 + wave;
  if (n < tile_end) {
    find_pages(0);
    load_keys(n);
    load_scales(n);
    load_values(n);
  }
  while (n < tile_end) {
    const int next = n + kPagedWaves;
    // Which of the tile's keys count, where it is not all of them.
    bool all = n * kKeys >= span.first && (n + 1) * kKeys <= span.len;
    bool has[kS];
#pragma unroll
    for (int s = 0; s < kS; ++s) {
      has[s] = page[s] >= 0;
      all = all && has[s];
    }
    float sc[kS][4];
#pragma unroll
    for (int s = 0; s < kS; ++s) {
      f32x4 c = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int k = 0; k < kKL; ++k) {
        if constexpr (k8) {
          c = mfma_16<FORMAT>(widen8<FORMAT>(kr[s][k].x, kr[s][k].y), qf[2 * k], c);
          c = mfma_16<FORMAT>(widen8<FORMAT>(kr[s][k].z, kr[s][k].w), qf[2 * k + 1], c);
        } else {
          c = mfma_16<FORMAT>(kr[s][k], qf[k], c);
        }
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float f = a.scale_log2e;
        if constexpr (k8) f *= dk[s][r];
        if constexpr (k8 && TYPE == TILEMIX_BF16) f = __builtin_amdgcn_ldexpf(f, -q_exp);
        sc[s][r] = c[r] * f;
      }
    }
    f32x4 dvc[kS];
    if constexpr (k8) {
#pragma unroll
      for (int s = 0; s < kS; ++s) dvc[s] = dv[s];
    }
    if (!all) {
#pragma unroll
      for (int s = 0; s < kS; ++s)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int t = n * kKeys + 16 * s + 4 * lq + r;
          const bool ok = has[s] && t >= span.first && t < span.len;
          sc[s][r] = ok ? sc[s][r] : ninf;
          if constexpr (k8) dvc[s][r] = ok ? dvc[s][r] : 0.0f;
          // What a slot behind the sequence holds may be a NaN, which a weight of 0 does not cancel.
          if constexpr (FORMAT != TILEMIX_INT8) {
#pragma unroll
            for (int w = 0; w < kVW; ++w) vr[s][r][w] = ok ? vr[s][r][w] : 0u;
          }
        }
    }
    // The next tile: its page ids, and its key rows into the registers of this one's.
    if (next < tile_end) {
      ++i;
      if ((i & (id_tiles - 1)) == 0) ids = load_ids(i);
      find_pages(i);
      load_keys(next);
    }
    // Softmax: the running max, normalizer and output move when the max or the values' exponent grows.
    float mt = sc[0][0];
#pragma unroll
    for (int s = 0; s < kS; ++s)
#pragma unroll
      for (int r = 0; r < 4; ++r) mt = fmaxf(mt, sc[s][r]);
    const float m_new = fmaxf(m, quad_rows_max(mt));
    int e_new = e;
    if constexpr (k8) {
      float vm = 0.0f;
#pragma unroll
      for (int s = 0; s < kS; ++s)
#pragma unroll
        for (int r = 0; r < 4; ++r) vm = fmaxf(vm, fabsf(dvc[s][r]));
      vm = quad_rows_max(vm);
      if (vm > 0.0f) e_new = max(e, __builtin_amdgcn_frexp_expf(vm));
    }
    if (__any(m_new > m || e_new > e)) {
      const float alpha = m == ninf ? 0.0f : __builtin_amdgcn_exp2f(m - m_new);
      z *= alpha;
      const float beta = k8 ? __builtin_amdgcn_ldexpf(alpha, e - e_new) : alpha;
#pragma unroll
      for (int c = 0; c < kC; ++c) acc[c] *= beta;
      m = m_new;
      e = e_new;
    }
    const float msub = m == ninf ? 0.0f : m - kShift<FORMAT>;
    uint2 hi[kS], lo[kS];
#pragma unroll
    for (int s = 0; s < kS; ++s) {
      float w[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float pr = __builtin_amdgcn_exp2f(sc[s][r] - msub);
        z += pr;
        w[r] = k8 ? pr * __builtin_amdgcn_ldexpf(dvc[s][r], -e) : pr;
      }
      split4<FORMAT>(w, hi[s], lo[s]);
    }
    // O^T += V^T P^T.
#pragma unroll
    for (int t = 0; t < kS / 2; ++t) {
      const uint4 ph = make_uint4(hi[2 * t].x, hi[2 * t].y, hi[2 * t + 1].x, hi[2 * t + 1].y);
      const uint4 pl = make_uint4(lo[2 * t].x, lo[2 * t].y, lo[2 * t + 1].x, lo[2 * t + 1].y);
#pragma unroll
      for (int c2 = 0; c2 < kC / 2; ++c2) {
        // Channels 2 c2 and 2 c2 + 1 of the lane, in FP16 or BF16, of its 8 keys.
        uint32_t x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const uint32_t (&row)[kVW] = vr[2 * t + j / 4][j % 4];
          if constexpr (!k8) x[j] = row[c2];
          else if constexpr (FORMAT == TILEMIX_E4M3) x[j] = c2 & 1 ? e4m3x2_to_half2<true>(row[c2 / 2]) : e4m3x2_to_half2<false>(row[c2 / 2]);
          else x[j] = row[c2 / 2];
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t v[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if constexpr (FORMAT == TILEMIX_INT8) {
              // A byte u of a code with the sign bit flipped reads as 1024 + 128 + code in 0x64uu.
              const uint32_t k = 2 * (c2 & 1) + h;
              const uint32_t pair = __builtin_amdgcn_perm(x[2 * j + 1], x[2 * j], 0x0c040c00u + k * 0x00010001u) ^ 0x64806480u;
              const half2_t bias = {(_Float16)-1152.0f, (_Float16)-1152.0f};
              v[j] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(half2_t, pair) + bias);
            } else {
              v[j] = __builtin_amdgcn_perm(x[2 * j + 1], x[2 * j], h ? 0x07060302u : 0x05040100u);
            }
          }
          const uint4 va = make_uint4(v[0], v[1], v[2], v[3]);
          const int c = 2 * c2 + h;
          acc[c] = mfma_16<FORMAT>(va, ph, acc[c]);
          acc[c] = mfma_16<FORMAT>(va, pl, acc[c]);
        }
      }
    }
    if (next < tile_end) {
      load_scales(next);
      load_values(next);
    }
    n = next;
  }

  // 5. The waves' results joined in LDS.
  z = quad_rows_sum(z);
  if (lq == 0) red_m[wave][l16] = m;
  if (lane == 0) red_e[wave] = e;
  __syncthreads();
  float mc = red_m[0][l16];
  int ec = red_e[0];
#pragma unroll
  for (int w = 1; w < kPagedWaves; ++w) {
    mc = fmaxf(mc, red_m[w][l16]);
    ec = max(ec, red_e[w]);
  }
  const float fw = m == ninf ? 0.0f : __builtin_amdgcn_exp2f(m - mc);
  if (lq == 0) red_z[wave][l16] = z * fw;
  const float fo = k8 ? __builtin_amdgcn_ldexpf(fw, e - ec) : fw;
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int c = 0; c < kC; ++c) osum[wave][l16][(4 * lq + r) * kC + c] = m == ninf ? 0.0f : acc[c][r] * fo;
  __syncthreads();
  const bool whole = ch.count == 1;
  for (int o = tid; o < heads * D; o += kPagedWaves * kWave) {
    const int g = o / D, c = o % D;
    float sum = 0.0f, zz = 0.0f;
#pragma unroll
    for (int w = 0; w < kPagedWaves; ++w) {
      sum += osum[w][g][c];
      zz += red_z[w][g];
    }
    if (whole) {
      const float x = zz == 0.0f ? 0.0f : k8 ? __builtin_amdgcn_ldexpf(sum / zz, ec) : sum / zz;
      static_cast<uint16_t*>(a.O)[((long long)b * a.Hq + hq0 + g) * D + c] = (uint16_t)float_to_bits<TYPE>(x);
    } else {
      a.part_o[((size_t)blockIdx.x * a.part_heads + g) * D + c] = sum;
    }
  }
  if (tid < heads) {
    float zz = 0.0f, mm = red_m[0][tid];
#pragma unroll
    for (int w = 0; w < kPagedWaves; ++w) {
      zz += red_z[w][tid];
      mm = fmaxf(mm, red_m[w][tid]);
    }
    if (whole) {
      if (a.lse)
        a.lse[(long long)b * a.Hq + hq0 + tid] =
            zz == 0.0f ? ninf : 0.69314718056f * (mm - kShift<FORMAT> + __builtin_amdgcn_logf(zz));
    } else {
      float* part = a.part_mze + ((size_t)blockIdx.x * a.part_heads + tid) * 3;
      part[0] = mm;
      part[1] = zz;
      part[2] = __builtin_bit_cast(float, ec);
    }
  }
  // Where the sequence's chunks are, for the join.
  if (a.segments && tid == 0 && ch.index == 0)
    reinterpret_cast<int2*>(a.segments)[(size_t)b * a.head_blocks + ch.head_block] = make_int2(ch.first_id, ch.count);
}

// One workgroup per (query head, sequence): thread (part, channel quad) joins every kParts-th chunk.
constexpr int kJoinThreads = 256;
template <int D, int TYPE, int FORMAT>
__global__ __launch_bounds__(kJoinThreads) void paged_join_kernel(PagedDecodeArgs a) {
  constexpr int kLanes = D / 4, kParts = kJoinThreads / kLanes, kWaves = kJoinThreads / kWave;
  constexpr int kAhead = 4;
  const int hq = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, wave = tid / kWave;
  const int G = a.Hq / a.pool.Hk, blocks = a.head_blocks / a.pool.Hk, hk = hq / G, g = hq % G;
  const int2 seg = reinterpret_cast<const int2*>(a.segments)[(size_t)b * a.head_blocks + hk * blocks + g / kPagedHeads];
  if (seg.y == 1) return;   // written already
  const int c4 = tid % kLanes, part = tid / kLanes;
  const float ninf = -__builtin_huge_valf();
  __shared__ f32x4 so[kParts][kLanes];
  __shared__ float sz[kParts], sm[kWaves], se[kWaves];
  auto row = [&](int i) { return (size_t)(seg.x + i) * a.part_heads + g % kPagedHeads; };
  auto exp_of = [&](const float* pm) { return __builtin_bit_cast(int, pm[2]); };
  // The largest max and exponent (a small whole number: exact in FP32) of all chunks.
  float m = ninf, ef = ninf;
  for (int i = tid; i < seg.y; i += kJoinThreads) {
    const float* pm = a.part_mze + 3 * row(i);
    m = fmaxf(m, pm[0]);
    ef = fmaxf(ef, (float)exp_of(pm));
  }
  m = wave_max(m);
  ef = wave_max(ef);
  if (tid % kWave == 0) {
    sm[wave] = m;
    se[wave] = ef;
  }
  __syncthreads();
  m = sm[0];
  ef = se[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) {
    m = fmaxf(m, sm[w]);
    ef = fmaxf(ef, se[w]);
  }
  const int e = (int)ef;
  float z = 0.0f;
  f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int i0 = part; i0 < seg.y; i0 += kParts * kAhead) {
    float f[kAhead], zi[kAhead];
    f32x4 oi[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int i = i0 + u * kParts;
      const float* pm = a.part_mze + 3 * row(min(i, seg.y - 1));
      oi[u] = *reinterpret_cast<const f32x4*>(a.part_o + row(min(i, seg.y - 1)) * D + 4 * c4);
      zi[u] = i < seg.y ? pm[1] : 0.0f;
      const bool some = i < seg.y && pm[0] != ninf;
      f[u] = some ? __builtin_amdgcn_exp2f(pm[0] - m) : 0.0f;
      z += zi[u] * f[u];
      if constexpr (is_8bit(FORMAT)) f[u] = __builtin_amdgcn_ldexpf(f[u], exp_of(pm) - e);
      oi[u] = some ? oi[u] : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) o += oi[u] * f[u];
  }
  so[part][c4] = o;
  if (c4 == 0) sz[part] = z;
  __syncthreads();
  if (tid < kLanes) {
    z = 0.0f;
    o = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int q = 0; q < kParts; ++q) {
      z += sz[q];
      o += so[q][tid];
    }
    const long long at = (long long)b * a.Hq + hq;
    uint32_t h[4];
#pragma unroll
    for (int r = 0; r < 4; ++r)
      h[r] = float_to_bits<TYPE>(z == 0.0f ? 0.0f : is_8bit(FORMAT) ? __builtin_amdgcn_ldexpf(o[r] / z, e) : o[r] / z);
    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.O) + at * D + 4 * tid) = make_uint2(h[0] | h[1] << 16, h[2] | h[3] << 16);
    if (tid == 0 && a.lse) a.lse[at] = z == 0.0f ? ninf : 0.69314718056f * (m - kShift<FORMAT> + __builtin_amdgcn_logf(z));
  }
}

}  // namespace

PagedDecodePlan plan_paged_decode(const PagedPool& p, int heads_q, int format) {
  const int G = heads_q / p.Hk;
  PagedDecodePlan pl{};
  pl.head_blocks = p.Hk * ((G + kPagedHeads - 1) / kPagedHeads);
  pl.part_heads = std::min(G, kPagedHeads);
  const int keys = tile_keys(format);
  const long long most = (((long long)p.max_pages << p.page_shift) + keys - 1) / keys;   // tiles of a sequence
  const long long segments = (long long)p.B * pl.head_blocks;
  pl.tiles = segments * most;
  pl.chunk_workgroups = kPagedWorkgroups;
  // Chunks hold kPagedWaves tiles at least; a sequence's last one is not full.
  pl.workgroups = std::min(pl.chunk_workgroups + segments, segments * ((most + kPagedWaves - 1) / kPagedWaves));
  pl.join = most > kPagedWaves;
  return pl;
}

hipError_t launch_paged_decode(const PagedDecodeArgs& a, const PagedDecodePlan& pl, int d, int type, int format,
                               hipStream_t stream) {
  return for_paged_types(d, type, format, [&](auto D, auto T, auto F) {
    hipLaunchKernelGGL((paged_decode_kernel<D(), T(), F()>), dim3((unsigned)pl.workgroups), dim3(kPagedWaves * kWave), 0, stream, a);
    if (pl.join)
      hipLaunchKernelGGL((paged_join_kernel<D(), T(), F()>), dim3(a.Hq, a.pool.B), dim3(kJoinThreads), 0,
                         stream, a);
    return hipGetLastError();
  });
}

}  // namespace tilemix
