// paged_decode.hip -- one decode step over the paged key/value cache.
//
// For query head hq of sequence b, over the tokens j attended to (the last `window`, or all, whose page
// exists): s_j = scale q . k_j, O = sum_j e^(s_j - m) v_j / sum_j e^(s_j - m), lse = m + ln of that sum.
//
//   paged_decode_kernel: as many workgroups of 4 waves as run at once, at most, share the tiles of the batch (see
//     Run); a workgroup has tiles of one or several (sequence, head block)s that follow one another.  In each of
//     them its waves stream tiles with a running (max, normalizer, output) of their own in registers; they are
//     joined in LDS, and the workgroup writes O, or a partial result where others have tiles of the same
//     sequence and heads.
//   paged_join_kernel: joins the partial results of one (sequence, query head) by their log-sum-exp.
//
// Bound: HBM.  Each cached row is read once per block of 16 query heads, with O(1) work per byte.
#include "paged_device.h"

#include <algorithm>

namespace tilemix {

namespace {

constexpr int kPagedWaves = 4;
constexpr int kCUs = 256;
// What it costs to begin and end a sequence and head block, in tiles.  (us, 64 sequences of 1 to 4000 keys, INT8, 8
// heads of d = 128: 3 tiles 58.6, 6 53.6, 9 54.6, 14 57.5.)
constexpr int kPartStart = 6;
constexpr int kPagedHeads = 16;                  // query heads on the columns of a matrix-core tile
// A tile is two slabs of 16 keys, of an MXFP4 cache, whose rows are half as long as an 8-bit one's, four: as many
// bytes, so that as many are on their way.  (Four slabs of an 8-bit cache leave two waves per SIMD instead of three: 32
// sequences of 64 to 8192 keys 34.9 us, with two slabs 30.9; 4 x 65536 keys 102.9 and 105.1.)
constexpr int tile_slabs(int format) { return is_4bit(format) ? 4 : 2; }
// Waves that a SIMD holds, by their registers (K and V rows of a tile, the output): workgroups per CU.  (MXFP4 with four at
// d = 64, some of whose variants spill then, us with four and with three: 32 sequences of 64 to 8192 keys, 32 / 8 heads, 19.4
// and 18.2; 16 of 700 to 20001, 16 / 4 heads, 17.2 and 15.7; 131072 keys, 28 / 4 heads, 21.8 and 20.2; 64 x 65536 keys,
// 16 / 4 heads, 240 and 240, in pages of 16 tokens 269 and 260; with two 19.1, 15.4, 18.3, 244 and 277.)
constexpr int resident_per_cu(int d, int format) { return d == 64 && !is_4bit(format) ? 4 : 3; }

// The tokens that a sequence's query attends to: first .. len - 1, of tiles tile0 .. .
template <int KEYS>   // of a tile
struct Span {
  int first = 0, len = 0, tile0 = 0, tiles = 0;
  Span() = default;
  __device__ __forceinline__ Span(const PagedDecodeArgs& a, int tokens) {
    const PagedPool& p = a.pool;
    len = min(max(tokens, 0), p.max_pages << p.page_shift);
    first = a.window > 0 ? max(len - a.window, 0) : 0;
    tile0 = first / KEYS;
    tiles = (len + KEYS - 1) / KEYS - tile0;
  }
  // Tiles as they are shared out: a sequence without tokens has one, so that it is written, too.
  __device__ __forceinline__ int share() const { return max(1, tiles); }
};

// A value that all lanes read from memory that nobody writes meanwhile, through the scalar path.
__device__ __forceinline__ int load_uniform(const int* p) {
  return *(const __attribute__((address_space(4))) int*)(uintptr_t)p;
}

// How the batch is cut into the workgroups' runs.  Sequences and head blocks are lined up, by sequence, then head block.
//   kPieces: each is cut into equal pieces, the fewest of `quota` tiles at most, and a workgroup takes one piece.
//   kRuns: each takes kPartStart units, for what it costs to begin and end one, and then a unit for each of its
//     tiles; workgroup w takes the tiles in units [w quota, (w + 1) quota).
//   kWhole: a workgroup takes `quota` of them, and none is shared by workgroups.
// kWhole is taken where that leaves no workgroup with more than 1.6 times the even share of tiles: memory is as busy with
// fewer waves, and what it costs to cut and join is saved (64 equal sequences of 4000 keys, INT8, 8 KV heads, d = 128,
// 90.7 us, cut into runs 100.7; 128 of them 173.3 and 187.8; at 2 times the share, 48 of them, 80.6 and 74.7).  Runs
// share the tiles evenly, pieces begin and end one sequence only: pieces are taken where their number fits the
// workgroups with at most kPartStart tiles more each than the even share (with up to twice the share 64 sequences of 1
// to 4000 keys took 67.3 us, in runs 57.5).  Every wave finds its place for itself: a lane takes a run of sequences.
enum { kPieces, kRuns, kWhole };

// n / d for 0 <= n < 2^31, d >= 1 and quotients below 2^20: an estimate in FP32, off by one at most, and a
// correction, in a third of the instructions of the compiler's division.
__device__ __forceinline__ int small_quotient(int n, int d) {
  const int q = (int)((float)n * __builtin_amdgcn_rcpf((float)d)), r = n - q * d;
  return q + (r >= d ? 1 : 0) - (r < 0 ? 1 : 0);
}
__device__ __forceinline__ int ceil_div(int n, int d) { return small_quotient(n + d - 1, d); }

// The largest of the lanes' x >= 0.
__device__ __forceinline__ int wave_max(int x) {
  x = max(x, dpp<0x111>(0, x));
  x = max(x, dpp<0x112>(0, x));
  x = max(x, dpp<0x114>(0, x));
  x = max(x, dpp<0x118>(0, x));
  x = max(x, dpp<0x142, 0xa>(0, x));
  x = max(x, dpp<0x143, 0xc>(0, x));
  return __builtin_amdgcn_readlane(x, kWave - 1);
}

template <int KEYS>
struct Run {
  int b = -1, head_block, unit;   // where it begins (unit, or piece: of its sequence's); b = -1: no tile is left
  int mode, quota;
  int total;                      // tiles of all sequences and head blocks
  __device__ __forceinline__ int units(int share) const {
    return mode == kWhole ? 1 : mode == kPieces ? ceil_div(share, quota) : kPartStart + share;
  }
  __device__ __forceinline__ Run(const PagedDecodeArgs& a, int w, int lane) {
    const int B = a.pool.B, per = (B + kWave - 1) / kWave, b0 = min(lane * per, B), b1 = min(b0 + per, B), W = gridDim.x;
    auto share = [&](int s) { return Span<KEYS>(a, a.pool.seqlens[s]).share(); };
    auto wave_total = [](int x) { return __builtin_amdgcn_readlane(wave_scan(x), kWave - 1); };
    // (Of up to 64 sequences, a lane's length is read once.)
    const int mine = b0 < b1 ? share(b0) : 0;
    auto over_lane = [&](auto&& f) {
      int sum = b0 < b1 ? f(mine) : 0;
      for (int s = b0 + 1; s < b1; ++s) sum += f(share(s));
      return sum;
    };
    mode = a.whole ? kWhole : kRuns;
    int own, all;
    if (mode == kWhole) {
      own = b1 - b0;
      all = B * a.head_blocks;
      // (For want of the lengths: half of the most.  By the first sequence's length, which the workgroup reads next, 64
      // sequences in page tables of 2048 slots took, INT8, 8 KV heads, d = 128: of 64 tokens 7.9 and 7.9 us, 200 11.1 and 11.4, 500
      // 16.7 and 16.1, 1000 27.1 and 27.2.)
      total = all * (a.whole / 2);
      quota = (int)a.div_workgroups.quot(all + W - 1);
    } else {
      int longest = 0;
      const int tiles = over_lane([&](int n) { longest = max(longest, n); return n; });
      total = wave_total(tiles) * a.head_blocks;
      const int even = max(kPagedWaves, (int)a.div_workgroups.quot(total + W - 1));
      longest = wave_max(longest);
      const int segments = B * a.head_blocks, each = (int)a.div_workgroups.quot(segments + W - 1);
      if (5ll * each * longest <= 8ll * even) {
        mode = kWhole;
        own = b1 - b0;
        all = segments;
        quota = each;
      } else if (segments <= W) {
        mode = kPieces;
        for (quota = even; quota <= even + kPartStart; quota += 2) {
          own = over_lane([&](int n) { return ceil_div(n, quota); });
          all = wave_total(own) * a.head_blocks;
          if (all <= W) break;
        }
        if (quota > even + kPartStart) mode = kRuns;
      }
      if (mode == kRuns) {
        own = tiles + kPartStart * (b1 - b0);
        all = total + kPartStart * B * a.head_blocks;
        quota = max(kPagedWaves, (int)a.div_workgroups.quot(all + W - 1));
      }
    }
    const int end = wave_scan(own), step = mode == kPieces ? 1 : quota;
    if ((long long)w * step >= all) return;
    const int u = w * step;
    int at = (end - own) * a.head_blocks, seq = 0, hb = 0, in = 0;
    const bool hit = u >= at && u < end * a.head_blocks;
    if (hit) {
      for (int s = b0; s < b1; ++s) {
        const int n = units(s == b0 ? mine : share(s)), next = at + n * a.head_blocks;
        if (u < next) {
          seq = s;
          hb = small_quotient(u - at, n);
          in = (u - at) - hb * n;
          break;
        }
        at = next;
      }
    }
    const int l = __builtin_ctzll(__ballot(hit));
    b = __builtin_amdgcn_readlane(seq, l);
    head_block = __builtin_amdgcn_readlane(hb, l);
    unit = __builtin_amdgcn_readlane(in, l);
  }
};

// A workgroup's part of one sequence and head block.  All members are the same in every lane.
template <int KEYS>
struct Part {
  Span<KEYS> span;
  int b = -1, head_block = 0;
  int lo = 0, hi = 0;          // its tiles, counted from the span's first: lo .. hi - 1 of span.share()
  int take = 0;                // the units that they are
  int step = 1;                // tiles of each workgroup that follows in the sequence and head block
  int tile0 = 0, end = 0;      // its tiles that hold tokens: tile0 .. end - 1
  int hk = 0, g0 = 0;          // KV head, first query head of the block among the KV head's
  Part() = default;
  // From unit `off` of the sequence and head block on, `left` units at most.
  __device__ __forceinline__ Part(const PagedDecodeArgs& a, int mode, int quota, int b_, int hb, int off, int left, const Span<KEYS>& sp)
      : span(sp), b(b_), head_block(hb) {
    const int n = span.share();
    hk = (int)a.div_blocks.quot(hb);
    g0 = (hb - hk * (int)a.div_blocks.d) * kPagedHeads;
    take = 1;
    hi = n;
    if (mode == kPieces) {
      step = ceil_div(n, ceil_div(n, quota));
      lo = off * step;
      hi = min(n, lo + step);
    } else if (mode == kRuns) {
      take = min(left, kPartStart + n - off);
      step = quota;
      lo = max(off - kPartStart, 0);
      hi = off + take - kPartStart;
    }
    tile0 = span.tile0 + lo;
    end = span.tile0 + min(span.tiles, hi);
  }
  __device__ __forceinline__ bool some() const { return hi > lo; }
  // The same in scalar registers, where the compiler lost track of it.
  __device__ __forceinline__ Part uniform() const {
    Part q = *this;
    for (int* x : {&q.span.first, &q.span.len, &q.span.tile0, &q.span.tiles, &q.b, &q.head_block, &q.lo, &q.hi, &q.take, &q.step, &q.tile0,
                   &q.end, &q.hk, &q.g0})
      *x = __builtin_amdgcn_readfirstlane(*x);
    return q;
  }
};

// A row's bytes.  `stream`: not kept in the caches, for batches of many bytes: 4 x 65536 keys of 8 INT8 heads (554 MB)
// 105.1 us, streamed 95.3; 131072 keys of 4 E4M3 heads (138 MB) 37.0 and 36.0; but 111 MB 30.9 and 31.4, 82 MB 21.4 and
// 22.6.  Not where a KV head has several blocks of query heads, each of which reads its rows: 8 x 32768 keys of
// one INT8 head, 32 query heads (69 MB) 30.5 us, streamed 35.6; of 64 query heads 28.0 and 31.0 (16384 keys, 35 MB); 16 x 65536
// keys (277 MB), 32 query heads, 78.3 and 89.5.  (Pages that sequences share count once for each, for want of
// a cheap way to know: 64 of 2500 to 3100 tokens of which they share 2048 55.6 us, streamed, as it is, 71.7.)
constexpr long long kStreamBytes = 128 << 20;
template <bool STREAM, typename V>
__device__ __forceinline__ V load_row(const char* p) {
  if constexpr (STREAM) return __builtin_nontemporal_load(reinterpret_cast<const V*>(p));
  return *reinterpret_cast<const V*>(p);
}
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Matrix-core products with 16-bit operands as the cache needs them: BF16 for a BF16 cache and for MXFP4, whose
// values are exact in BF16, else FP16 (8-bit codes are exact in FP16).
constexpr int operand_type(int format) { return format == TILEMIX_BF16 || is_4bit(format) ? TILEMIX_BF16 : TILEMIX_FP16; }
template <int FORMAT>
__device__ __forceinline__ f32x4 mfma_16(uint4 x, uint4 y, f32x4 c) {
  if constexpr (operand_type(FORMAT) == TILEMIX_BF16)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(as_half8(x), as_half8(y), c, 0, 0, 0);
}

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

// The scale operand of the conversions of byte b of w.  They take its exponent field and leave the other bits alone, so
// a rotation by 8 b + 9 to the right is enough.
__device__ __forceinline__ float exponent_scale(uint32_t w, int b) {
  return __builtin_bit_cast(float, __builtin_amdgcn_alignbit(w, w, 8 * b + 9));
}

// The lanes' x as CTRL moves them; every lane has a source.
template <int CTRL>
__device__ __forceinline__ int dpp_all(int x) {
  return __builtin_amdgcn_update_dpp(0, x, CTRL, 0xf, 0xf, true);
}

// x of the lane that holds the other piece of the same head (PAIRED): lane ^ 8.
__device__ __forceinline__ float other_piece(float x) {
  return __builtin_bit_cast(float, dpp_all<0x128>(__builtin_bit_cast(int, x)));
}

// x of lane L of the four lanes that agree in lane / 4.
template <int L>
__device__ __forceinline__ uint32_t quad_lane(uint32_t x) {
  return (uint32_t)dpp_all<L * 0x55>((int)x);
}

// p = 2^(s - m) is taken against the running max m, and so is the normalizer z = sum p.  The weights of the codes
// are p dV 2^-x (p 2^-x for 16 and 4 bits): x = 0 for a BF16 cache and MXFP4, -15 for an FP16 one, and e - 15 for an 8-bit
// one, where 2^e is above every value scale dV so far.  They stay at 2^15 at most, and are handed to the matrix cores as
// two 16-bit pieces: FP16 pieces hold them to 2^-22 of themselves, and to 2^-40 of the largest possible
// weight where they are small; BF16 pieces to 2^-16, with FP32's range.  One piece alone (2^-12 or
// 2^-9) would add as much error as the output's own rounding.  m and x go through the joins side by side:
// m + x is another number in FP32 where |m| is large, by more than 1 from 2^25 on, and a weight of 2^16 is no FP16
// number any more; and z, which knows nothing of x, loses nothing to a value's size.  e starts at kExpMin, that of the
// smallest subnormal scale, 2^-149: values near BF16's smallest are weighted like any others.
constexpr int kExpMin = -148;
constexpr int kKeyTop = 13;   // the largest exponent of MXFP4 keys in FP16: 6 2^13 is the largest of them
template <int FORMAT>
constexpr int kHeadroom = operand_type(FORMAT) == TILEMIX_BF16 ? 0 : 15;

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// Two 16-bit pieces of two weights.
template <int FORMAT>
__device__ __forceinline__ void split2(float w0, float w1, uint32_t& hi, uint32_t& lo) {
  using V = std::conditional_t<operand_type(FORMAT) == TILEMIX_BF16, bf16x2, half2v>;
  const V h = __builtin_convertvector((f32x2{w0, w1}), V);
  const V l = __builtin_convertvector((f32x2{w0 - (float)h[0], w1 - (float)h[1]}), V);
  hi = __builtin_bit_cast(uint32_t, h);
  lo = __builtin_bit_cast(uint32_t, l);
}

// One BF16 piece of two weights (see split2): the first, or else the second.
__device__ __forceinline__ uint32_t own_piece(float w0, float w1, bool first) {
  const uint32_t h = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{w0, w1}), bf16x2)) & (first ? 0u : ~0u);
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{w0 - __builtin_bit_cast(float, h << 16),
                                                                     w1 - __builtin_bit_cast(float, h & 0xffff0000u)}), bf16x2));
}

// Scores are computed transposed, S^T = K Q^T: a slab's 16 keys on the rows, the query heads on the columns
// of a 16x16 product, so that lane (l16, lq) = (lane % 16, lane / 16) receives keys 4 lq + r (r < 4) of
// head l16.  For the pair of slabs 2 t, 2 t + 1 these are the eight keys that the B operand of
// O^T += V^T P^T wants in that lane, so P stays in registers.  The A operand V^T wants the same keys of
// channel row l16; row i of product c is given channel i D / 16 + c, so that a lane reads D / 16
// adjacent channels of a key at once and pairs the keys by byte permutes: no transposed copy of V is
// kept, and a row can be appended to a page as it is.
template <int D>
struct DecodeShared {
  float m[kPagedWaves][kPagedHeads], z[kPagedWaves][kPagedHeads];
  int x[kPagedWaves];
  __align__(16) float o[kPagedWaves][kPagedHeads][D + 4];   // padded rows
};

// Two variants of MXFP4 (an MXFP4 tile has as many bytes as the others' and twice the work, and what bounds it beside the
// memory is how many instructions a wave issues: one in some 8 cycles, scalar ones too):
// PAIRED: KV heads of up to 8 query heads.  Half of the 16 columns would be padding: columns h and h + 8 both belong to head
// h and carry the two pieces of its weights, and of an FP16 query, which add up to the scores of both.  Half of the
// products of O^T += V^T P^T are spared.
// ONE_PAGE: pages hold whole tiles, so that a tile's rows lie one behind the other.  The addresses of four slabs are 200 of 780
// instructions of a tile: 8 x 65536 keys (FP16, BF16 queries) 111 and 109 us without, 106 and 103 with it.
template <int D, int TYPE, int FORMAT, bool STREAM, bool PAIRED, bool ONE_PAGE>
__device__ __forceinline__ void decode_run(const PagedDecodeArgs& a, const Run<16 * tile_slabs(FORMAT)>& run, DecodeShared<D>& shared) {
  constexpr int kS = tile_slabs(FORMAT), kKeys = 16 * kS;
  typedef Span<kKeys> Span;
  typedef Part<kKeys> Part;
  constexpr int kBytes = kElemBytes<FORMAT>;
  constexpr bool k8 = is_8bit(FORMAT), k4 = is_4bit(FORMAT);
  constexpr int kRow = kRowBytes<D, FORMAT>, kScaleRow = kScaleBytes<D, FORMAT>;
  constexpr int kKL = k4 ? 1 : kRow / 64;          // loads of a key row per lane, 16 bytes each (MXFP4, d = 64: 8)
  constexpr int kC = D / 16;                       // channels of a lane's value row: output products
  constexpr int kVW = k4 ? 1 : kC * kBytes / 4;    // dwords of them
  constexpr int kQ = D / 32;                       // score products per slab
  constexpr bool kRelative = k4 && TYPE == TILEMIX_FP16 && !PAIRED;   // keys relative to the largest exponent of their tile (see 4.)
  const PagedPool& p = a.pool;
  const int tid = threadIdx.x, lane = tid & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int l16 = lane & 15, lq = lane >> 4, column = PAIRED ? l16 & 7 : l16;   // column: query head of the block
  const float ninf = -__builtin_huge_valf();
  auto& red_m = shared.m;
  auto& red_z = shared.z;
  auto& red_x = shared.x;
  auto& osum = shared.o;

  const int quota = __builtin_amdgcn_readfirstlane(run.quota), mode = __builtin_amdgcn_readfirstlane(run.mode);
  int left = mode == kPieces ? 1 : quota;   // units
  Part cur;
  {
    const int b = __builtin_amdgcn_readfirstlane(run.b);
    if (b < 0) return;
    cur = Part(a, mode, quota, b, __builtin_amdgcn_readfirstlane(run.head_block), __builtin_amdgcn_readfirstlane(run.unit), left,
               Span(a, load_uniform(p.seqlens + b)));
    if (!cur.some()) return;
  }
  // The wave's first tile of a part, if f tiles of the workgroup's run lie before it: tile f + t goes to wave
  // (f + t) % kPagedWaves, so that the waves have the same number over all parts.
  auto first_tile = [&](const Part& q, int f) { return q.tile0 + ((wave - f) & (kPagedWaves - 1)); };

  // 1. Page ids of the wave's tiles n, n + kPagedWaves, .. of a part, 64 at a time: lane (i, j) holds the j-th of
  //    the 2^per_shift pages of tile i.
  const int per_shift = max(0, (kKeys == 64 ? 6 : 5) - p.page_shift);
  auto load_ids = [&](const Part& q, int n0) {
    const int n = n0 + (lane >> per_shift) * kPagedWaves;
    const int e = (n * kKeys >> p.page_shift) + (lane & ((1 << per_shift) - 1));
    int id = -1;
    if (n < q.end && e < p.max_pages && (e << p.page_shift) < q.span.len) id = p.table[q.b * p.stride_table + e];
    return id;
  };
  const int id_tiles = kWave >> per_shift;

  // 2. One tile in registers.  Where a wave has no tile to request it requests some all the same (see 4.), a few
  //    cache lines of page 0: every lane's offset is 0.
  uint4 kr[kS][kKL];
  uint32_t vr[kS][4][kVW];
  f32x4 dk[kS], dv[kS];
  // MXFP4: words with the exponents of key l16 and of key 4 lq + l16 % 4 (d = 64: of two keys).  All rows and exponents are loaded as
  // whole words: of a narrower one the compiler clears the upper bits as soon as it is loaded, and waits for it there.
  uint32_t ek[kS], ev[kS];
  const int key_byte = kScaleRow == 4 ? lq : 2 * (l16 & 1) + (lq >> 1);   // of the lane's channels in ek
  constexpr int kPages = ONE_PAGE ? 1 : kS;
  int page[kPages];                                // per slab, of the tile that was requested last
  const char* poolK = static_cast<const char*>(p.K);
  const char* poolV = static_cast<const char*>(p.V);
  const uint32_t k_lane = l16 * kRow + (k4 ? kRow / 4 : 16) * lq, v_lane = 4 * lq * kRow + (k4 ? l16 * (kRow / 16) & ~3 : l16 * (kRow / 16));
  auto find_pages = [&](int ids, int i) {
    const int at = (i & (id_tiles - 1)) << per_shift;
#pragma unroll
    for (int s = 0; s < kPages; ++s) {
      const int id = __builtin_amdgcn_readlane(ids, at + (16 * s >> p.page_shift));
      page[s] = id < p.pages ? id : -1;
    }
  };
  // Row of slab s of tile n in its page, or in page 0 where there is none: it is masked.  slab_at: bytes from the pool's start,
  // of rows of row_bytes and pages `stride` elements of `elem` bytes apart.  (Not for the rows of 16 bits and 8: with it 16-bit
  // kernels have their arguments fetched over and over; 1000 keys of two heads, FP16, d = 64, 5.96 us, without 5.76.)
  auto slab_row = [&](int hk, int n, int s) { return (hk << p.page_shift) + ((n * kKeys + 16 * s) & ((1 << p.page_shift) - 1)); };
  auto slab_at = [&](int hk, int n, int s, long long stride, int elem, int row_bytes) {
    const int from = ONE_PAGE ? 0 : s;
    return elem * (max(page[from], 0) * stride) + (long long)slab_row(hk, n, from) * row_bytes + (s - from) * 16 * row_bytes;
  };
  auto load_keys = [&](int hk, int n, bool some) {
    const uint32_t k_off = some ? k_lane : 0u, s_off = some ? 16u * lq : 0u;
#pragma unroll
    for (int s = 0; s < kS; ++s) {
      const char* base = k4 ? poolK + slab_at(hk, n, s, p.stride_k, kBytes, kRow)
                            : poolK + kBytes * (max(page[s % kPages], 0) * p.stride_k + (long long)slab_row(hk, n, s) * D);
      if constexpr (k4 && D == 64) {
        const u32x2 x = load_row<STREAM, u32x2>(base + k_off);
        kr[s][0] = make_uint4(x[0], x[1], 0, 0);
      } else {
#pragma unroll
        for (int i = 0; i < kKL; ++i) kr[s][i] = __builtin_bit_cast(uint4, load_row<STREAM, u32x4>(base + 64 * i + k_off));
      }
    }
    if constexpr (k8) {
#pragma unroll
      for (int s = 0; s < kS; ++s)
        dk[s] = *reinterpret_cast<const f32x4*>(static_cast<const char*>(p.dK) + slab_at(hk, n, s, p.stride_dk, 4, 4) + s_off);
    }
    if constexpr (k4) {
#pragma unroll
      for (int s = 0; s < kS; ++s)
        ek[s] = *reinterpret_cast<const uint32_t*>(static_cast<const char*>(p.dK) + slab_at(hk, n, s, p.stride_dk, 1, kScaleRow) +
                                                   (some ? l16 * kScaleRow & ~3u : 0u));
    }
  };
  auto load_values = [&](int hk, int n, bool some) {
    const uint32_t v_off = some ? v_lane : 0u, s_off = some ? 16u * lq : 0u;
    if constexpr (k8) {
#pragma unroll
      for (int s = 0; s < kS; ++s)
        dv[s] = *reinterpret_cast<const f32x4*>(static_cast<const char*>(p.dV) + slab_at(hk, n, s, p.stride_dv, 4, 4) + s_off);
    }
    if constexpr (k4) {
#pragma unroll
      for (int s = 0; s < kS; ++s) {
        ev[s] = *reinterpret_cast<const uint32_t*>(static_cast<const char*>(p.dV) + slab_at(hk, n, s, p.stride_dv, 1, kScaleRow) +
                                                   (some ? kScaleRow * (4 * lq + l16 % 4) & ~3u : 0u));
      }
    }
#pragma unroll
    for (int s = 0; s < kS; ++s) {
      const char* base = k4 ? poolV + slab_at(hk, n, s, p.stride_v, kBytes, kRow)
                            : poolV + kBytes * (max(page[s % kPages], 0) * p.stride_v + (long long)slab_row(hk, n, s) * D);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const char* at = base + r * kRow + v_off;
        if constexpr (kVW == 4) {
          const u32x4 x = load_row<STREAM, u32x4>(at);
          vr[s][r][0] = x[0]; vr[s][r][1] = x[1]; vr[s][r][2] = x[2]; vr[s][r][3] = x[3];
        } else if constexpr (kVW == 2) {
          const u32x2 x = load_row<STREAM, u32x2>(at);
          vr[s][r][0] = x[0]; vr[s][r][1] = x[1];
        } else {
          vr[s][r][0] = load_row<STREAM, uint32_t>(at);
        }
      }
    }
  };
  uint4 qf[kQ];
  auto load_query = [&](const Part& q) {
    const int G = a.group, heads = min(kPagedHeads, G - q.g0);
    const char* row = static_cast<const char*>(a.Q) + 2 * (q.b * a.q_stride + (long long)(q.hk * G + q.g0 + min(column, heads - 1)) * D);
#pragma unroll
    for (int i = 0; i < kQ; ++i) qf[i] = ld_global_16(row + 2 * (k4 ? D / 4 * lq + 8 * i : k8 ? 64 * (i / 2) + 16 * lq + 8 * (i % 2) : 32 * i + 8 * lq));
  };

  int f = 0, i = 0, n = first_tile(cur, 0);
  int ids = load_ids(cur, n);
  load_query(cur);
  find_pages(ids, 0);
  __builtin_amdgcn_sched_barrier(0);
  load_keys(cur.hk, n, n < cur.end);
  __builtin_amdgcn_sched_barrier(0);
  load_values(cur.hk, n, n < cur.end);
  __builtin_amdgcn_sched_barrier(0);
  for (;;) {
    const int G = a.group, heads = min(kPagedHeads, G - cur.g0), hq0 = cur.hk * G + cur.g0;
    cur = cur.uniform();
    n = __builtin_amdgcn_readfirstlane(n);
    left = __builtin_amdgcn_readfirstlane(left);
    // The part that follows, so that its first tiles are requested behind the last ones of this.
    Part next;
    const bool whole_head = cur.head_block + 1 == a.head_blocks;
    bool more = left > cur.take && !(whole_head && cur.b + 1 == p.B);
    if (more) {
      next = Part(a, mode, quota, cur.b + (whole_head ? 1 : 0), whole_head ? 0 : cur.head_block + 1, 0, left - cur.take,
                  whole_head ? Span(a, load_uniform(p.seqlens + cur.b + 1)) : cur.span);
      more = next.some();
    }
    const int f_next = f + cur.hi - cur.lo, n_next = first_tile(next, f_next);
    const int ids_next = load_ids(next, n_next);

    // 3. Query rows as the B operand of the score products: lane (head l16, lq) holds the channels that it
    //    reads of a key row.  BF16 queries against 8-bit codes are brought to FP16 by a power of two per
    //    head, 2^q_exp: the largest to [2^14, 2^15), so that what FP16 cannot hold lies below 2^-39 of it.  2^109 is
    //    enough: it brings BF16's smallest number to FP16's, so that nothing is lost, and what takes it back in
    //    f_head is then no subnormal number (for scales of 2^-17 and more).
    float f_head = a.scale_log2e;   // score of a product, in log2 units, before the key's scale
    {
      const uint32_t some = column < heads ? ~0u : 0u;
  #pragma unroll
      for (int i = 0; i < kQ; ++i) qf[i] = make_uint4(qf[i].x & some, qf[i].y & some, qf[i].z & some, qf[i].w & some);
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
        const int q_exp = min(15 - __builtin_amdgcn_frexp_expf(quad_rows_max(amax)), 109);
        f_head = __builtin_amdgcn_ldexpf(f_head, -q_exp);
  #pragma unroll
        for (int i = 0; i < kQ; ++i) {
          uint32_t w[8];
  #pragma unroll
          for (int e = 0; e < 8; ++e) w[e] = float_to_bits<TILEMIX_FP16>(__builtin_amdgcn_ldexpf(x[i][e], q_exp));
          qf[i] = make_uint4(w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16, w[6] | w[7] << 16);
        }
      }
      if constexpr (PAIRED && TYPE == TILEMIX_FP16) {   // FP16's 11 bits are two BF16 numbers of 8 and 3
  #pragma unroll
        for (int i = 0; i < kQ; ++i) {
          const uint32_t w[4] = {qf[i].x, qf[i].y, qf[i].z, qf[i].w};
          uint32_t h[4];
  #pragma unroll
          for (int e = 0; e < 4; ++e) {
            h[e] = own_piece(bits_to_float<TILEMIX_FP16>(w[e] & 0xffffu), bits_to_float<TILEMIX_FP16>(w[e] >> 16), l16 < 8);
          }
          qf[i] = make_uint4(h[0], h[1], h[2], h[3]);
        }
      }
    }

    // 4. The wave's tiles.  m: running max (log2 units); x: the weights' power of two; z: this lane's share of the
    //    normalizer; acc: output.  Loads complete in order, and a wait counts the younger ones, so rows are requested in the
    //    same order and number on every way to a wait: the keys and their scales once the scores are
    //    formed, the values and theirs after P V, into the registers that these leave, whether there is
    //    another tile in this part, in the next one, or none.
    float m = ninf, z = 0.0f;
    int x = (k8 ? kExpMin : 0) - kHeadroom<FORMAT>;
    f32x4 acc[kC];
  #pragma unroll
    for (int c = 0; c < kC; ++c) acc[c] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const bool none = n >= cur.end;
    while (n < cur.end) {
      // Which of the tile's keys count, where it is not all of them.
      bool all = n * kKeys >= cur.span.first && (n + 1) * kKeys <= cur.span.len;
      uint32_t has = ONE_PAGE && page[0] >= 0 ? (1u << kS) - 1 : 0u;
  #pragma unroll
      for (int s = 0; s < (ONE_PAGE ? 0 : kS); ++s) has |= page[s] >= 0 ? 1u << s : 0u;
      all = all && has == (1u << kS) - 1;
      // FP16 queries take MXFP4 keys in FP16: code 2^(e - top + kKeyTop), top the largest exponent of a key that counts, so that
      // what FP16 cannot hold lies below 2^-38 of 2^top.  (As two BF16 pieces, which lose nothing, they took twice the products
      // and 16 registers more, which spilled: 8 x 65536 keys 119 us.)  A NaN among them is one in all scores.  What takes a
      // score back to its size is a factor up to 1 and, for keys beyond 2^13, a power of two for the score itself: as
      // one factor it is infinite for scales of 6 and more beside BF16's largest numbers.
      float f_tile = f_head;
      uint32_t top = 0;
      if constexpr (kRelative) {
        if (!all) {
  #pragma unroll
          for (int s = 0; s < kS; ++s) {
            const int t = n * kKeys + 16 * s + l16;
            ek[s] = (has >> s & 1) && t >= cur.span.first && t < cur.span.len ? ek[s] : 0u;
          }
        }
  #pragma unroll
        for (int s = 0; s < kS; ++s) ek[s] = ek[s] >> 8 * key_byte & 0xffu;
        uint32_t e = ek[0];
  #pragma unroll
        for (int s = 1; s < kS; ++s) e = max(e, ek[s]);
        top = (uint32_t)wave_max((int)e);
        f_tile = top == kBlockNaN ? __builtin_nanf("") : __builtin_amdgcn_ldexpf(f_head, min((int)top - 127 - kKeyTop, 0));
      }
      float sc[kS][4];
  #pragma unroll
      for (int s = 0; s < kS; ++s) {
        f32x4 c = {0.0f, 0.0f, 0.0f, 0.0f};
        if constexpr (k4) {
          const float scale = kRelative ? block_scale(max(ek[s] + 127 + kKeyTop, top) - top) : exponent_scale(ek[s], key_byte);
          const uint32_t w[4] = {kr[s][0].x, kr[s][0].y, kr[s][0].z, kr[s][0].w};
  #pragma unroll
          for (int k = 0; k < kQ; ++k) {
            constexpr int kType = kRelative ? TILEMIX_FP16 : TILEMIX_BF16;
            c = mfma_16<kType>(mx_values8<kType>(w[k], scale), qf[k], c);
          }
        }
  #pragma unroll
        for (int k = 0; k < (k4 ? 0 : kKL); ++k) {
          if constexpr (k8) {
            c = mfma_16<FORMAT>(widen8<FORMAT>(kr[s][k].x, kr[s][k].y), qf[2 * k], c);
            c = mfma_16<FORMAT>(widen8<FORMAT>(kr[s][k].z, kr[s][k].w), qf[2 * k + 1], c);
          } else {
            c = mfma_16<FORMAT>(kr[s][k], qf[k], c);
          }
        }
        if constexpr (PAIRED && TYPE == TILEMIX_FP16) {
  #pragma unroll
          for (int r = 0; r < 4; ++r) c[r] += other_piece(c[r]);
        }
        // Scores are scaled and rounded before the max and the exponent see them.
  #pragma unroll
        for (int r = 0; r < 4; ++r) sc[s][r] = c[r] * (k8 ? f_head * dk[s][r] : f_tile);
      }
      if constexpr (kRelative) {
        if (top > 127 + kKeyTop) {
  #pragma unroll
          for (int s = 0; s < kS; ++s)
  #pragma unroll
            for (int r = 0; r < 4; ++r) sc[s][r] = __builtin_amdgcn_ldexpf(sc[s][r], (int)top - 127 - kKeyTop);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      const bool here = n + kPagedWaves < cur.end;
      const int to = here ? n + kPagedWaves : n_next, hk = here ? cur.hk : next.hk;
      const bool some = here || n_next < next.end;
      if (here) {
        ++i;
        if ((i & (id_tiles - 1)) == 0) {
          ids = load_ids(cur, to);
          asm volatile("; wait for them here" : "+v"(ids));   // not on the other ways, where rows are in flight
        }
      } else {
        i = 0;
        ids = ids_next;
        asm volatile("; and here for the next part's" : "+v"(ids));
      }
      find_pages(ids, i);
      load_keys(hk, to, some);
      if (!all) {
  #pragma unroll
        for (int s = 0; s < kS; ++s)
  #pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int t = n * kKeys + 16 * s + 4 * lq + r;
            const bool ok = (has >> s & 1) && t >= cur.span.first && t < cur.span.len;
            sc[s][r] = ok ? sc[s][r] : ninf;
            if constexpr (k8) dv[s][r] = ok ? dv[s][r] : 0.0f;
            // What a slot behind the sequence holds may be a NaN, which a weight of 0 does not cancel.
            if constexpr (k4) {   // (d = 64: the other key of the word has its own lane)
              if (l16 % 4 == r) ev[s] = ok ? ev[s] : 0u;
            } else if constexpr (FORMAT != TILEMIX_INT8) {
  #pragma unroll
              for (int w = 0; w < kVW; ++w) vr[s][r][w] = ok ? vr[s][r][w] : 0u;
            }
          }
      }
      // Softmax: normalizer and output move when the max or the value scales' exponent grows.
      float mt = sc[0][0];
  #pragma unroll
      for (int s = 0; s < kS; ++s)
  #pragma unroll
        for (int r = 0; r < 4; ++r) mt = fmaxf(mt, sc[s][r]);
      const float m_new = fmaxf(m, quad_rows_max(mt));
      int x_new = x;
      if constexpr (k8) {
        float vm = 0.0f;
  #pragma unroll
        for (int s = 0; s < kS; ++s)
  #pragma unroll
          for (int r = 0; r < 4; ++r) vm = fmaxf(vm, fabsf(dv[s][r]));
        vm = quad_rows_max(vm);
        if (vm > 0.0f) x_new = max(x, __builtin_amdgcn_frexp_expf(vm) - kHeadroom<FORMAT>);
      }
      if (__any(m_new > m || x_new > x)) {
        const float alpha = m == ninf ? 0.0f : __builtin_amdgcn_exp2f(m - m_new);
        const float beta = k8 ? __builtin_amdgcn_ldexpf(alpha, x - x_new) : alpha;
        z *= alpha;
  #pragma unroll
        for (int c = 0; c < kC; ++c) acc[c] *= beta;
        m = m_new;
        x = x_new;
      }
      // No finite score so far: p = 2^(-inf - 0) = 0, not a NaN.
      const float sub = m == ninf ? 0.0f : m;
      // O^T += V^T P^T.
#pragma unroll
      for (int t = 0; t < kS; t += 2) {   // a pair of slabs
      uint2 hi[2], lo[2];
  #pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int s = t + u;
        float w[4];
  #pragma unroll
        for (int r = 0; r < 4; ++r) {
          w[r] = __builtin_amdgcn_exp2f(sc[s][r] - sub);
          z += w[r];
          if constexpr (k8) w[r] *= __builtin_amdgcn_ldexpf(dv[s][r], -x);
          else if constexpr (FORMAT == TILEMIX_FP16) w[r] *= 0x1p15f;
        }
        if constexpr (PAIRED) {
          hi[u].x = own_piece(w[0], w[1], l16 < 8);
          hi[u].y = own_piece(w[2], w[3], l16 < 8);
        } else {
          split2<FORMAT>(w[0], w[1], hi[u].x, lo[u].x);
          split2<FORMAT>(w[2], w[3], hi[u].y, lo[u].y);
        }
      }
      const uint4 ph = make_uint4(hi[0].x, hi[0].y, hi[1].x, hi[1].y), pl = make_uint4(lo[0].x, lo[0].y, lo[1].x, lo[1].y);
      auto row = [&](int j) -> const uint32_t (&)[kVW] { return vr[t + j / 4][j % 4]; };   // of the lane's key j < 8
      auto add = [&](int c, const uint32_t (&v)[4]) {
        const uint4 va = make_uint4(v[0], v[1], v[2], v[3]);
        acc[c] = mfma_16<FORMAT>(va, ph, acc[c]);
        if constexpr (!PAIRED) acc[c] = mfma_16<FORMAT>(va, pl, acc[c]);
      };
      if constexpr (k4) {
        // Two channels of a key in a byte: widened, with the key's scale of the lane's channels, then paired.
        float ve[8];
  #pragma unroll
        for (int u = 0; u < 2; ++u) {
          const uint32_t w[4] = {quad_lane<0>(ev[t + u]), quad_lane<1>(ev[t + u]), quad_lane<2>(ev[t + u]), quad_lane<3>(ev[t + u])};
  #pragma unroll
          for (int r = 0; r < 4; ++r) ve[4 * u + r] = exponent_scale(w[r], l16 * kC / 32 + (kScaleRow == 2 ? 2 * (r & 1) : 0));
        }
        // d = 64: a lane's two bytes are one half of its word, and those of two keys are brought into one.
        uint32_t codes[8];
        if constexpr (D == 64) {
          const uint32_t pick = l16 & 1 ? 0x07060302u : 0x05040100u;
  #pragma unroll
          for (int j = 0; j < 4; ++j) codes[j] = __builtin_amdgcn_perm(row(2 * j + 1)[0], row(2 * j)[0], pick);
        } else {
  #pragma unroll
          for (int j = 0; j < 8; ++j) codes[j] = row(j)[0];
        }
  #pragma unroll
        for (int c = 0; c < kC; c += 2) {
          uint32_t v[2][4];
  #pragma unroll
          for (int j = 0; j < 4; ++j) {
            uint32_t x[2];
  #pragma unroll
            for (int u = 0; u < 2; ++u) {
              const uint32_t w = D == 64 ? codes[j] : codes[2 * j + u];
              const int byte = D == 64 ? c / 2 + 2 * u : c / 2;
              const float scale = ve[2 * j + u];
              x[u] = byte == 0 ? mx_values<TILEMIX_BF16, 0>(w, scale) : byte == 1 ? mx_values<TILEMIX_BF16, 1>(w, scale)
                   : byte == 2 ? mx_values<TILEMIX_BF16, 2>(w, scale) : mx_values<TILEMIX_BF16, 3>(w, scale);
            }
            v[0][j] = __builtin_amdgcn_perm(x[1], x[0], 0x05040100u);
            v[1][j] = __builtin_amdgcn_perm(x[1], x[0], 0x07060302u);
          }
          add(c, v[0]);
          add(c + 1, v[1]);
        }
      } else if constexpr (FORMAT == TILEMIX_E4M3) {
        // Channels c and c + 1 of two keys in one word, then two conversions.
  #pragma unroll
        for (int c = 0; c < kC; c += 2) {
          uint32_t v[2][4];
  #pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint32_t w = __builtin_amdgcn_perm(row(2 * j + 1)[c / 4], row(2 * j)[c / 4], c & 2 ? 0x07030602u : 0x05010400u);
            v[0][j] = e4m3x2_to_half2<false>(w);
            v[1][j] = e4m3x2_to_half2<true>(w);
          }
          add(c, v[0]);
          add(c + 1, v[1]);
        }
      } else {
  #pragma unroll
        for (int c = 0; c < kC; ++c) {
          uint32_t v[4];
  #pragma unroll
          for (int j = 0; j < 4; ++j) {
            if constexpr (FORMAT == TILEMIX_INT8) {
              // A byte u of a code with the sign bit flipped reads as 1024 + 128 + code in 0x64uu.
              const uint32_t pair = __builtin_amdgcn_perm(row(2 * j + 1)[c / 4], row(2 * j)[c / 4],
                                                          0x0c040c00u + (uint32_t)(c & 3) * 0x00010001u) ^ 0x64806480u;
              const half2v bias = {(_Float16)-1152.0f, (_Float16)-1152.0f};
              v[j] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(half2v, pair) + bias);
            } else {
              v[j] = __builtin_amdgcn_perm(row(2 * j + 1)[c / 2], row(2 * j)[c / 2], c & 1 ? 0x07060302u : 0x05040100u);
            }
          }
          add(c, v);
        }
      }
      }
      __builtin_amdgcn_sched_barrier(0);   // not ahead of P V: their registers are in use
      load_values(hk, to, some);
      n += kPagedWaves;
    }
    if (none) {   // the wave's registers hold nothing of this part
      i = 0;
      ids = ids_next;
      find_pages(ids, 0);
      load_keys(next.hk, n_next, n_next < next.end);
      __builtin_amdgcn_sched_barrier(0);
      load_values(next.hk, n_next, n_next < next.end);
    }
    __builtin_amdgcn_sched_barrier(0);
    if (more) load_query(next);

    // 5. The waves' results joined in LDS.
    z = quad_rows_sum(z);
    if (lq == 0) red_m[wave][l16] = m;
    if (lane == 0) red_x[wave] = x;
    __syncthreads();
    float top = red_m[0][l16];
    int xx = red_x[0];
  #pragma unroll
    for (int w = 1; w < kPagedWaves; ++w) {
      top = fmaxf(top, red_m[w][l16]);
      xx = max(xx, red_x[w]);
    }
    const float fz = m == ninf ? 0.0f : __builtin_amdgcn_exp2f(m - top), fw = k8 ? __builtin_amdgcn_ldexpf(fz, x - xx) : fz;
    if (lq == 0) red_z[wave][l16] = z * fz;
  #pragma unroll
    for (int r = 0; r < 4; ++r)
  #pragma unroll
      for (int c = 0; c < kC; ++c) osum[wave][l16][(4 * lq + r) * kC + c] = m == ninf ? 0.0f : acc[c][r] * fw;
    __syncthreads();
    const bool whole = cur.lo == 0 && cur.hi == cur.span.share();
    // Partial results: of the workgroup's first part in row 2 w, of one behind others in row 2 w + 1 (it is the
    // last, and has its sequence's first tile).
    const int part_row = (int)blockIdx.x * 2 + (f != 0 ? 1 : 0);
    for (int o = tid; o < heads * (D / 4); o += kPagedWaves * kWave) {
      const int g = o / (D / 4), c = o % (D / 4) * 4;
      f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
      float zz = 0.0f;
  #pragma unroll
      for (int w = 0; w < kPagedWaves; ++w) {
        sum += *reinterpret_cast<const f32x4*>(&osum[w][g][c]);
        if constexpr (PAIRED) sum += *reinterpret_cast<const f32x4*>(&osum[w][g + 8][c]);
        zz += red_z[w][g];
      }
      if (whole) {
        uint32_t h[4];
  #pragma unroll
        for (int r = 0; r < 4; ++r) h[r] = float_to_bits<TYPE>(zz == 0.0f ? 0.0f : __builtin_amdgcn_ldexpf(sum[r] / zz, xx));
        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.O) + ((long long)cur.b * a.Hq + hq0 + g) * D + c) =
            make_uint2(h[0] | h[1] << 16, h[2] | h[3] << 16);
      } else {
        *reinterpret_cast<f32x4*>(a.part_o + ((size_t)part_row * a.part_heads + g) * D + c) = sum;
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
          a.lse[(long long)cur.b * a.Hq + hq0 + tid] =
              zz == 0.0f ? ninf : 0.69314718056f * (mm + __builtin_amdgcn_logf(zz));
      } else {
        reinterpret_cast<float4*>(a.part_mzx)[(size_t)part_row * a.part_heads + tid] = make_float4(mm, zz, __int_as_float(xx), 0.0f);
      }
    }
    // For the join: the first row, and how many workgroups there are from this one on.
    if (a.segments && tid == 0 && cur.lo == 0) {
      const int beyond = cur.span.share() - cur.hi;   // tiles of the workgroups that follow
      reinterpret_cast<int2*>(a.segments)[(size_t)cur.b * a.head_blocks + cur.head_block] =
          make_int2(part_row, 1 + ceil_div(beyond, cur.step));
    }
    if (!more) return;
    left -= cur.take;
    cur = next;
    f = f_next;
    n = n_next;
    __syncthreads();   // the LDS is used again
  }
}

template <int D, int TYPE, int FORMAT, bool PAIRED, bool ONE_PAGE>
__global__ __launch_bounds__(kPagedWaves * kWave) __attribute__((amdgpu_waves_per_eu(resident_per_cu(D, FORMAT))))
void paged_decode_kernel(PagedDecodeArgs a) {
  __shared__ DecodeShared<D> shared;
  constexpr int kKeys = 16 * tile_slabs(FORMAT);
  const Run<kKeys> run(a, blockIdx.x, threadIdx.x & (kWave - 1));
  // (Two copies of the body: a branch at each request would make the waits count loads that were not issued.)
  const long long bytes = (long long)__builtin_amdgcn_readfirstlane(run.total) * (kKeys * 2 * kRowBytes<D, FORMAT>);
  if (bytes >= kStreamBytes && a.head_blocks == a.pool.Hk) decode_run<D, TYPE, FORMAT, true, PAIRED, ONE_PAGE>(a, run, shared);
  else decode_run<D, TYPE, FORMAT, false, PAIRED, ONE_PAGE>(a, run, shared);
}

// op over the lanes that agree in lane % LANES (8, 16 or 32).
template <int LANES, typename T, typename OP>
__device__ __forceinline__ T across(T x, OP op) {
  auto bits = [](T y) { return __builtin_bit_cast(int, y); };
  auto join = [&](int y, int z) { return op(__builtin_bit_cast(T, y), __builtin_bit_cast(T, z)); };
  if constexpr (LANES == 8) x = join(bits(x), dpp<0x128>(bits(x), bits(x)));   // lane ^ 8
  if constexpr (LANES <= 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(bits(x), bits(x), false, false);
    x = join((int)r[0], (int)r[1]);
  }
  const auto r = __builtin_amdgcn_permlane32_swap(bits(x), bits(x), false, false);
  return join((int)r[0], (int)r[1]);
}

// One workgroup per (query head, sequence, CHANNELS channels): thread (part, channel quad) joins every kParts-th row
// with a running max and power of two of its own.  kNoExp: below every row's power.
constexpr int kNoExp = -1024;
constexpr int kJoinThreads = 256;
template <int D, int TYPE, int CHANNELS>
__global__ __launch_bounds__(kJoinThreads) void paged_join_kernel(PagedDecodeArgs a) {
  constexpr int kLanes = CHANNELS / 4, kParts = kJoinThreads / kLanes, kWaves = kJoinThreads / kWave, kAhead = 4;
  const int hq = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
  const int hk = (int)a.div_group.quot(hq), g = hq - hk * a.group, blocks = (int)a.div_blocks.d;
  const int2 seg = reinterpret_cast<const int2*>(a.segments)[(size_t)b * a.head_blocks + hk * blocks + g / kPagedHeads];
  if (seg.y == 1) return;   // written already
  const int c4 = tid % kLanes, part = tid / kLanes, c0 = blockIdx.z * CHANNELS;
  const float ninf = -__builtin_huge_valf();
  __shared__ f32x4 so[kWaves][kLanes];
  __shared__ float sz[kWaves], sm[kWaves];
  __shared__ int sx[kWaves];
  // Row i of the partial results: the first may be its workgroup's second row, the others are first rows.
  auto row = [&](int i) { return (size_t)(i == 0 ? seg.x : (seg.x & ~1) + 2 * i) * a.part_heads + g % kPagedHeads; };
  const float4* mzx = reinterpret_cast<const float4*>(a.part_mzx);
  float m = ninf, z = 0.0f;
  int x = kNoExp;
  f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int i0 = part; i0 < seg.y; i0 += kParts * kAhead) {
    float4 ri[kAhead];
    f32x4 oi[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const size_t r = row(min(i0 + u * kParts, seg.y - 1));
      ri[u] = mzx[r];
      oi[u] = *reinterpret_cast<const f32x4*>(a.part_o + r * D + c0 + 4 * c4);
    }
    float top = m;
    int xx = x;
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      top = fmaxf(top, ri[u].x);
      xx = max(xx, __float_as_int(ri[u].z));
    }
    const float f = m == ninf ? 0.0f : __builtin_amdgcn_exp2f(m - top);
    z *= f;
    o *= __builtin_amdgcn_ldexpf(f, x - xx);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (i0 + u * kParts >= seg.y) break;
      // (A row without a finite score may hold a NaN as its normalizer.)
      const float fu = ri[u].x == ninf ? 0.0f : __builtin_amdgcn_exp2f(ri[u].x - top);
      z += ri[u].y * fu;
      o += oi[u] * __builtin_amdgcn_ldexpf(fu, __float_as_int(ri[u].z) - xx);
    }
    m = top;
    x = xx;
  }
  // A wave's parts are joined by lane exchanges, the waves in LDS.
  auto larger = [](auto x, auto y) { return x > y ? x : y; };
  auto plus = [](float x, float y) { return x + y; };
  float top = across<kLanes>(m, larger);
  int xx = across<kLanes>(x, larger);
  const float f = m == ninf ? 0.0f : __builtin_amdgcn_exp2f(m - top), fo = __builtin_amdgcn_ldexpf(f, x - xx);
  z = across<kLanes>(z * f, plus);
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = across<kLanes>(o[i] * fo, plus);
  const int wave = tid / kWave;
  if (tid % kWave < kLanes) so[wave][c4] = o;
  if (tid % kWave == 0) {
    sz[wave] = z;
    sm[wave] = top;
    sx[wave] = xx;
  }
  __syncthreads();
  if (tid < CHANNELS) {
    top = ninf;
    xx = kNoExp;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      top = fmaxf(top, sm[w]);
      xx = max(xx, sx[w]);
    }
    z = 0.0f;
    float y = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float fw = sm[w] == ninf ? 0.0f : __builtin_amdgcn_exp2f(sm[w] - top);
      z += sz[w] * fw;
      y += so[w][tid / 4][tid % 4] * __builtin_amdgcn_ldexpf(fw, sx[w] - xx);
    }
    const long long at = (long long)b * a.Hq + hq;
    static_cast<uint16_t*>(a.O)[at * D + c0 + tid] = (uint16_t)float_to_bits<TYPE>(z == 0.0f ? 0.0f : __builtin_amdgcn_ldexpf(y / z, xx));
    if (tid == 0 && c0 == 0 && a.lse) a.lse[at] = z == 0.0f ? ninf : 0.69314718056f * (top + __builtin_amdgcn_logf(z));
  }
}

}  // namespace

PagedDecodePlan plan_paged_decode(const PagedPool& p, int heads_q, int d, int format, int window) {
  const int G = heads_q / p.Hk, keys = 16 * tile_slabs(format);
  PagedDecodePlan pl{};
  pl.head_blocks = p.Hk * ((G + kPagedHeads - 1) / kPagedHeads);
  pl.part_heads = std::min(G, kPagedHeads);
  long long most = (((long long)p.max_pages << p.page_shift) + keys - 1) / keys;   // tiles of a sequence
  if (window > 0) most = std::min<long long>(most, (window + keys - 2LL) / keys + 1);
  const long long segments = (long long)p.B * pl.head_blocks;
  pl.units = segments * (most + kPartStart);
  const bool mx = is_4bit(format);
  // A tile of MXFP4 has twice the keys: two workgroups per CU keep the memory as busy as three where few sequences and
  // heads are cut, and leave fewer partial results.  us with three and with two, d = 128: 131072 keys, 28 / 4 heads, 27.6 and
  // 25.5; 32 sequences of 64 to 8192 keys, 32 / 8 heads, 25.3 and 24.6; 8 x 65536 keys, 64 / 8 heads, 98.2 and 96.5; but 64 of 1000
  // to 30000 keys 107 and 109, 128 of 1 to 4000 34.7 and 36.9; d = 64 32 of 64 to 8192 18.3 and 19.2.
  const long long resident = kCUs * (mx && d == 128 && segments <= kCUs ? 2 : resident_per_cu(d, format));
  // Where sequences cannot be long none is split whatever their lengths, and no second launch joins them.  How long,
  // depends on how many workgroups that leaves; us without and with a split, INT8, 8 KV heads, d = 128:
  //   16 tiles     1 sequence of 250 keys 7.7 and 9.5; 8 of 1000 keys 15.2 and 12.7
  //   32 from 128  16 of 1000 keys 15.4 and 16.1, 24 15.6 and 17.8; 16 of 1500 keys 19.9 and 17.8
  //   64 from 192  24 of 2000 keys 25.7 and 25.7, 32 28.3 and 33.3, 64 47.7 and 49.6; 24 of 4000 keys 45.4 and 40.9
  //   32 where workgroups take several: 128 of 1 to 2000 keys 75.4 and 65.5, of 1 to 1000 41.0 and 40.1
  // The same limits for the others: FP16 8 of 1000 14.7 and 13.8, 24 of 1000 19.5 and 23.5, 16 of 1500 23.4 and 23.2, 32 of
  // 2000 42.8 and 47.8, 24 of 4000 69.5 and 66.7 (but 128 of 1 to 1000 68.0 and 58.3); INT8, d = 64 24 of 1000 12.8 and
  // 13.8, 16 of 1500 16.4 and 14.0, 32 of 2000 20.0 and 20.6, 24 of 4000 35.2 and 27.0.
  // MXFP4's tiles, of 64 keys, us on the GPU (what a call takes is at the host's 11 us without the second launch and 15
  // with it): 1 sequence of 500 keys 9.5 and 10.6, of 1000 13.0 and 10.6; 16 of 1000 11.7 and 13.6, of 1900 17.0 and 16.3;
  // 24 of 1000 11.9 and 15.5, of 1900 18.8 and 21.2, of 500 to 4000 26.7 and 20.1; 32 of 1900 20.3 and 23.7, of 100 to 1900 16.9
  // and 16.0, of 4000 34.3 and 37.7, of 500 to 4000 27.9 and 24.6; 64 of 1900 30.7 and 33.1, of 4000 55.3 and 59.5; 128 of 2000
  // 62.0 and 64.1.
  const long long limit = segments < kCUs / 2 ? 16
                        : segments < kCUs * 3 / 4 ? (mx ? 16 : 32)
                        : segments > resident || (mx && segments < kCUs * 3 / 2) ? 32 : 64;
  pl.whole = most <= limit ? (int)most : 0;
  pl.workgroups = std::min<long long>(resident,
                                      pl.whole ? segments : (segments * most + kPagedWaves - 1) / kPagedWaves);
  return pl;
}

hipError_t launch_paged_decode(PagedDecodeArgs a, const PagedDecodePlan& pl, int d, int type, int format, hipStream_t stream) {
  a.group = a.Hq / a.pool.Hk;
  a.div_group = FastDiv(a.group);
  a.div_blocks = FastDiv(pl.head_blocks / a.pool.Hk);
  a.div_workgroups = FastDiv((uint32_t)pl.workgroups);
  return for_paged_types(d, type, format, [&](auto D, auto T, auto F) {
    const dim3 workgroups((unsigned)pl.workgroups), threads(kPagedWaves * kWave);
    auto go = [&](auto PAIRED, auto ONE_PAGE) {
      hipLaunchKernelGGL((paged_decode_kernel<D(), T(), F(), PAIRED(), ONE_PAGE()>), workgroups, threads, 0, stream, a);
    };
    if constexpr (is_4bit(F())) {
      const bool paired = a.group <= 8, one_page = 1 << a.pool.page_shift >= 16 * tile_slabs(F());
      if (paired && one_page) go(std::true_type{}, std::true_type{});
      else if (paired) go(std::true_type{}, std::false_type{});
      else if (one_page) go(std::false_type{}, std::true_type{});
      else go(std::false_type{}, std::false_type{});
    } else {
      go(std::false_type{}, std::false_type{});
    }
    if (pl.whole) return hipGetLastError();
    // All channels in a workgroup where there are many, most of them with nothing to join; 32 of them, and so more parts
    // at a time, where there are few or a sequence may have many rows (one has at most as many as there are
    // workgroups for a head block).  us, 32 and all channels, sequences of up to 4000 keys, INT8, 32 / 8 heads of d = 128:
    // 8 sequences 12.6 and 13.0, 16 20.3 and 19.7, 64 54.9 and 51.6, 128 105.9 and 101.2; one of 32000 keys 20.5 and 23.6.
    const dim3 grid(a.Hq, a.pool.B);
    if ((long long)a.Hq * a.pool.B >= 512 && pl.workgroups <= 256 * pl.head_blocks)
      hipLaunchKernelGGL((paged_join_kernel<D(), T(), D()>), grid, dim3(kJoinThreads), 0, stream, a);
    else
      hipLaunchKernelGGL((paged_join_kernel<D(), T(), 32>), dim3(grid.x, grid.y, D() / 32), dim3(kJoinThreads), 0, stream, a);
    return hipGetLastError();
  });
}

}  // namespace tilemix
