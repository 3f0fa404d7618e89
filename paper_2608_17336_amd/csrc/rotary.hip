// rotary.hip -- rotary positions on Q and K (bandwidth-bound).
//
// Pair i < r / 2 of a head at position p is turned by the angle p f_i and stretched by g:
//   (y1, y2) = g (x1 cos - x2 sin, x2 cos + x1 sin),
// (x1, x2) being channels (i, i + r / 2) or (2 i, 2 i + 1); channels from r on stay as they are.  `inverse` turns by
// -p f_i: the transposed map, which is the gradient of the other.
//
// An angle of a far position has more bits than FP32: it is reduced to a quarter turn in two FP64 numbers, and the sine and
// cosine of what is left, at most an eighth of a turn, are Taylor sums in FP32.  That is some 45 instructions, so a
// workgroup does it once for each (token, pair) and leaves both in LDS for all heads.
#include "paged_device.h"

#include <algorithm>

namespace tilemix {

namespace {

constexpr int kRotaryThreads = 256;
// Heads that a lane requests at a time.  (us at 1, 2, 4 and 8: 196 million BF16 elements, half of each head turned, 146, 146,
// 153 and 163; 4 x 8192 tokens of 64/8 heads, d = 128, 212, 207, 222 and 241.)
constexpr int kRowsAhead = 2;
// Results of this many bytes and more, and their inputs, pass the caches by: the same two 146 and 129, 207 and 189.  But a reader
// finds less in the caches: sequences of 512 tokens, 32 / 8 heads, d = 128, 126 MB 51.3 and 47.9, with their prefill 184 and 190;
// 147 MB 58.7 and 55.3, 211 and 214; 189 MB 73.5 and 70.0, 272 and 272; 336 MB 127 and 122, 463 and 459.
constexpr long long kStreamBytes = 160 << 20;
constexpr int kMaxTokens = 8;        // of a workgroup
constexpr int kGridShift = 23;       // a launch has less than 2^32 threads in x: 2^23 workgroups, and the others in y

// cos and sin of p f, p a whole number.  The product and its turns are each a sum of two FP64 numbers, and so is 1 / (2 pi):
// rounded to one, the turns of position 2^31 were off by up to 2^-24, where a result near 0 has no such room.  What is
// left of whole turns is then off by 2^-52.  |a| <= pi / 4: the first terms left out are below 2^-32.
__device__ __forceinline__ float2 cos_sin(int p, double f) {
#pragma clang fp contract(off)   // (a product whose rounding `low` takes up again must be rounded)
  constexpr double kTurn = 0.15915494309189535, kTurnLow = -9.839338337591243e-18;
  const double t = p * f, turns = t * kTurn;
  const double low = fma(t, kTurn, -turns) + fma(t, kTurnLow, fma((double)p, f, -t) * kTurn);
  const double quarters = (turns - rint(turns) + low) * 4.0, n = rint(quarters);
  const float a = (float)(quarters - n) * 1.57079632679489662f, b = a * a;
  float s = fmaf(b, -1.0f / 39916800, 1.0f / 362880);
  s = fmaf(b, s, -1.0f / 5040);
  s = fmaf(b, s, 1.0f / 120);
  s = fmaf(b, s, -1.0f / 6);
  s = fmaf(b * a, s, a);
  float c = fmaf(b, -1.0f / 3628800, 1.0f / 40320);
  c = fmaf(b, c, -1.0f / 720);
  c = fmaf(b, c, 1.0f / 24);
  c = fmaf(b, c, -0.5f);
  c = fmaf(b, c, 1.0f);
  const int k = (int)n & 3;
  const float x = k & 1 ? s : c, y = k & 1 ? c : s;
  return make_float2(k == 1 || k == 2 ? -x : x, k >= 2 ? -y : y);
}

// How many of the n numbers v[0 .. n - 1], which do not fall, are <= x: 64 are looked at at a time.  (Where they do
// fall the answer is some number of 0 .. n.)
__device__ __forceinline__ int wave_count(const int* v, int n, int x, int lane) {
  int lo = 0;
  while (n > 0) {
    const int step = (n + kWave - 1) / kWave, at = (lane + 1) * step - 1;
    const int full = __popcll(__ballot(at < n && v[lo + at] <= x));
    lo += full * step;
    n = min(step - 1, n - full * step);
  }
  return lo;
}

// Position of packed row i, or a negative number where it has none.  All lanes of a wave ask for the same row.
__device__ __forceinline__ int row_position(const RotaryArgs& a, int i, int lane) {
  if (i >= a.total) return -1;
  if (a.positions) return a.positions[i];
  if (!a.cu) {
    const int b = (int)a.div_len.quot(i);
    return (int)max((long long)a.seqlens[b] - (int)a.div_len.d + (i - b * (int)a.div_len.d), -1ll);
  }
  const int b = min(wave_count(a.cu + 1, a.batch, i, lane), a.batch - 1);
  const int from = min(max(a.cu[b], 0), a.total), to = min(max(a.cu[b + 1], from), a.total);
  return i < from || i >= to ? -1 : (int)max((long long)a.seqlens[b] - (to - from) + (i - from), -1ll);
}

template <int V>
struct Vec;
template <>
struct Vec<8> {
  typedef uint32_t t __attribute__((ext_vector_type(4)));
};
template <>
struct Vec<4> {
  typedef uint32_t t __attribute__((ext_vector_type(2)));
};
template <>
struct Vec<2> {
  typedef uint32_t t;
};
template <>
struct Vec<1> {
  typedef uint16_t t;
};

// V values of TYPE as FP32, and back.
template <int TYPE, int V>
__device__ __forceinline__ void unpack(typename Vec<V>::t v, float (&x)[V]) {
  uint16_t h[V];
  __builtin_memcpy(h, &v, 2 * V);
#pragma unroll
  for (int i = 0; i < V; ++i) x[i] = bits_to_float<TYPE>(h[i]);
}
template <int TYPE, int V>
__device__ __forceinline__ typename Vec<V>::t pack(const float (&x)[V]) {
  uint16_t h[V];
#pragma unroll
  for (int i = 0; i < V; ++i) h[i] = (uint16_t)float_to_bits<TYPE>(x[i]);
  typename Vec<V>::t v;
  __builtin_memcpy(&v, h, 2 * V);
  return v;
}

// A head of d channels is d / (2 V) units of two vectors of V channels: where pairs are r / 2 apart, the two halves of V
// pairs, then two adjacent vectors behind r; else two vectors d / 2 apart, each of V / 2 pairs or behind r.  A lane
// takes one unit of every step-th head of one token.
template <bool STREAM, typename T>
__device__ __forceinline__ T load(const uint16_t* p) {
  if constexpr (STREAM) return __builtin_nontemporal_load(reinterpret_cast<const T*>(p));
  return *reinterpret_cast<const T*>(p);
}
template <bool STREAM, typename T>
__device__ __forceinline__ void store(uint16_t* p, T x) {
  if constexpr (STREAM) __builtin_nontemporal_store(x, reinterpret_cast<T*>(p));
  else *reinterpret_cast<T*>(p) = x;
}

template <int TYPE, bool HALF, int V, bool STREAM>
__global__ __launch_bounds__(kRotaryThreads) void rotary_kernel(RotaryArgs a) {
  typedef typename Vec<V>::t Vt;
  __shared__ float2 turn[kMaxTokens * 64];
  __shared__ int where[kMaxTokens];
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
  const int d = a.d, r = a.r, pairs = r / 2, tokens = 1 << a.token_shift, first = (blockIdx.x + (blockIdx.y << kGridShift)) << a.token_shift;
  for (int t = wave; t < tokens; t += kRotaryThreads / kWave) {
    const int p = row_position(a, first + t, lane);
    if (lane == 0) where[t] = p;
  }
  __syncthreads();
  for (int k = tid; k < tokens * pairs; k += kRotaryThreads) {
    const int t = (int)a.div_pairs.quot(k), i = k - t * pairs;
    const float2 cs = cos_sin(where[t], a.inv_freq[i]);
    turn[k] = make_float2(cs.x * a.magnitude, a.inverse ? -cs.y * a.magnitude : cs.y * a.magnitude);
  }
  __syncthreads();

  const int unit_shift = a.unit_shift, u = tid & ((1 << unit_shift) - 1), group = tid >> unit_shift;
  const int token = group & (tokens - 1), h0 = group >> a.token_shift, step = (kRotaryThreads >> unit_shift) >> a.token_shift;
  if (where[token] < 0) return;
  const long long row = first + token;
  // The unit's vectors, and which of them turn.
  int c[2];
  bool turns[2];
  if constexpr (HALF) {
    const int n = pairs / V;
    turns[0] = turns[1] = u < n;
    c[0] = u < n ? u * V : r + (u - n) * 2 * V;
    c[1] = u < n ? c[0] + pairs : c[0] + V;
  } else {
    c[0] = u * V;
    c[1] = c[0] + d / 2;
    turns[0] = c[0] < r;
    turns[1] = c[1] < r;
  }
  const bool moves[2] = {turns[0] || !a.in_place, turns[1] || !a.in_place};
  float2 cs[V];   // of the pairs, those of the first vector first
  if constexpr (HALF) {
#pragma unroll
    for (int i = 0; i < V; ++i) cs[i] = turns[0] ? turn[token * pairs + c[0] + i] : make_float2(1.0f, 0.0f);
  } else {
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int i = 0; i < V / 2; ++i)
        cs[j * (V / 2) + i] = turns[j] ? turn[token * pairs + c[j] / 2 + i] : make_float2(1.0f, 0.0f);
  }
  const int heads = a.Hq + a.Hk;
  auto from = [&](int h) {
    return h < a.Hq ? static_cast<const uint16_t*>(a.Q) + row * a.q_stride + h * d
                    : static_cast<const uint16_t*>(a.K) + row * a.k_stride + (h - a.Hq) * d;
  };
  auto to = [&](int h) {
    return h < a.Hq ? static_cast<uint16_t*>(a.Q_out) + row * a.q_out_stride + h * d
                    : static_cast<uint16_t*>(a.K_out) + row * a.k_out_stride + (h - a.Hq) * d;
  };
  for (int h = h0; h < heads; h += step * kRowsAhead) {
    Vt v[kRowsAhead][2];
#pragma unroll
    for (int k = 0; k < kRowsAhead; ++k)
      if (h + k * step < heads) {
        const uint16_t* p = from(h + k * step);
#pragma unroll
        for (int j = 0; j < 2; ++j)
          if (moves[j]) v[k][j] = load<STREAM, Vt>(p + c[j]);
      }
#pragma unroll
    for (int k = 0; k < kRowsAhead; ++k) {
      if (h + k * step >= heads) break;
      uint16_t* p = to(h + k * step);
      float x[2][V], y[2][V];
#pragma unroll
      for (int j = 0; j < 2; ++j) unpack<TYPE, V>(v[k][j], x[j]);
      if constexpr (HALF) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
          y[0][i] = x[0][i] * cs[i].x - x[1][i] * cs[i].y;
          y[1][i] = x[1][i] * cs[i].x + x[0][i] * cs[i].y;
        }
      } else {
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int i = 0; i < V / 2; ++i) {
            const float2 w = cs[j * (V / 2) + i];
            y[j][2 * i] = x[j][2 * i] * w.x - x[j][2 * i + 1] * w.y;
            y[j][2 * i + 1] = x[j][2 * i + 1] * w.x + x[j][2 * i] * w.y;
          }
      }
#pragma unroll
      for (int j = 0; j < 2; ++j)   // (what does not turn is moved as it is, whatever it holds)
        if (moves[j]) store<STREAM, Vt>(p + c[j], turns[j] ? pack<TYPE, V>(y[j]) : v[k][j]);
    }
  }
}

}  // namespace

hipError_t launch_rotary(RotaryArgs a, int type, bool half, hipStream_t stream) {
  // Channels of a vector: the most that the pairs' distance allows.
  int v = 8;
  while ((half ? a.r / 2 : a.r) % v) v /= 2;
  const int units = a.d / (2 * v);
  a.unit_shift = 0;
  while ((1 << a.unit_shift) < units) ++a.unit_shift;
  const int groups = kRotaryThreads >> a.unit_shift, heads = a.Hq + a.Hk;
  a.token_shift = 0;
  while ((2 << a.token_shift) <= std::min(groups, kMaxTokens) && (groups >> a.token_shift) * kRowsAhead > 2 * heads &&
         a.total >> a.token_shift > 1024)
    ++a.token_shift;
  a.div_pairs = FastDiv((uint32_t)(a.r / 2));
  const unsigned workgroups = (unsigned)(((long long)a.total + (1 << a.token_shift) - 1) >> a.token_shift);
  const dim3 grid(std::min(workgroups, 1u << kGridShift), (workgroups + (1u << kGridShift) - 1) >> kGridShift);
  auto go = [&](auto T, auto H, auto V) {
    if (V() == 8 && 2LL * a.total * heads * a.d >= kStreamBytes)
      hipLaunchKernelGGL((rotary_kernel<T(), H(), V(), V() == 8>), grid, dim3(kRotaryThreads), 0, stream, a);
    else
      hipLaunchKernelGGL((rotary_kernel<T(), H(), V(), false>), grid, dim3(kRotaryThreads), 0, stream, a);
    return hipGetLastError();
  };
  using std::integral_constant;
  auto by_layout = [&](auto T) {
    if (half) {
      if (v == 8) return go(T, std::true_type{}, integral_constant<int, 8>{});
      if (v == 4) return go(T, std::true_type{}, integral_constant<int, 4>{});
      if (v == 2) return go(T, std::true_type{}, integral_constant<int, 2>{});
      return go(T, std::true_type{}, integral_constant<int, 1>{});
    }
    if (v == 8) return go(T, std::false_type{}, integral_constant<int, 8>{});
    if (v == 4) return go(T, std::false_type{}, integral_constant<int, 4>{});
    return go(T, std::false_type{}, integral_constant<int, 2>{});
  };
  return type == TILEMIX_BF16 ? by_layout(integral_constant<int, TILEMIX_BF16>{}) : by_layout(integral_constant<int, TILEMIX_FP16>{});
}

}  // namespace tilemix
