// paged_decode.hip -- one decode step over the paged key/value cache.
//
// For query head hq of sequence b, over the tokens j attended to (the last `window`, or all, whose page
// exists): s_j = scale q . k_j, O = sum_j e^(s_j - m) v_j / sum_j e^(s_j - m), lse = m + ln of that sum.
//
// One workgroup per (sequence, query head).  Its waves take tokens in turn, the lanes of a wave the
// channels; each wave keeps a running (max, normalizer, output), joined in LDS at the end.
#include "paged_device.h"

namespace tilemix {

namespace {

constexpr int kPagedWaves = 4;

__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) x += __shfl_xor(x, off, kWave);
  return x;
}

template <int D, int TYPE, int FORMAT>
__global__ __launch_bounds__(kPagedWaves * kWave) void paged_decode_kernel(PagedDecodeArgs a) {
  constexpr int kPer = D / kWave;
  const PagedPool& p = a.pool;
  const int hq = blockIdx.x, b = blockIdx.y, hk = hq / (a.Hq / p.Hk);
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave, c = lane * kPer;
  __shared__ float sm[kPagedWaves], sz[kPagedWaves], so[kPagedWaves][D];
  const uint16_t* q = static_cast<const uint16_t*>(a.Q) + b * a.q_stride + hq * D + c;
  float qx[kPer], o[kPer], m = -__builtin_huge_valf(), z = 0.0f;
#pragma unroll
  for (int e = 0; e < kPer; ++e) {
    qx[e] = bits_to_float<TYPE>(q[e]);
    o[e] = 0.0f;
  }
  const int len = min(max(p.seqlens[b], 0), p.max_pages << p.page_shift);
  const int first = a.window > 0 ? max(len - a.window, 0) : 0;
  auto channel = [](const void* base, long long at) {
    if constexpr (FORMAT == TILEMIX_INT8) return (float)static_cast<const int8_t*>(base)[at];
    else if constexpr (FORMAT == TILEMIX_E4M3)
      return (float)__builtin_amdgcn_cvt_f32_fp8(static_cast<const uint8_t*>(base)[at], 0);
    else return bits_to_float<FORMAT>(static_cast<const uint16_t*>(base)[at]);
  };
  for (int j = first + wave; j < len; j += kPagedWaves) {
    const Slot s = find_slot(p, b, j);
    if (s.page < 0) continue;
    const int row = (hk << p.page_shift) + s.slot;
    float dot = 0.0f;
#pragma unroll
    for (int e = 0; e < kPer; ++e) dot += qx[e] * channel(p.K, s.page * p.stride_k + (long long)row * D + c + e);
    float f = a.scale_log2e, dv = 1.0f;
    if constexpr (is_8bit(FORMAT)) {
      f *= p.dK[s.page * p.stride_dk + row];
      dv = p.dV[s.page * p.stride_dv + row];
    }
    const float sc = wave_sum(dot) * f, mn = fmaxf(m, sc);
    const float alpha = m == mn ? 1.0f : __builtin_amdgcn_exp2f(m - mn);
    const float pr = sc == -__builtin_huge_valf() ? 0.0f : __builtin_amdgcn_exp2f(sc - mn);
    z = z * alpha + pr;
#pragma unroll
    for (int e = 0; e < kPer; ++e)
      o[e] = o[e] * alpha + pr * dv * channel(p.V, s.page * p.stride_v + (long long)row * D + c + e);
    m = mn;
  }
  if (lane == 0) {
    sm[wave] = m;
    sz[wave] = z;
  }
#pragma unroll
  for (int e = 0; e < kPer; ++e) so[wave][c + e] = o[e];
  __syncthreads();
  float mm = sm[0];
#pragma unroll
  for (int w = 1; w < kPagedWaves; ++w) mm = fmaxf(mm, sm[w]);
  float zz = 0.0f, f[kPagedWaves];
#pragma unroll
  for (int w = 0; w < kPagedWaves; ++w) {
    f[w] = sm[w] == -__builtin_huge_valf() ? 0.0f : __builtin_amdgcn_exp2f(sm[w] - mm);
    zz += sz[w] * f[w];
  }
  const float inv = zz == 0.0f ? 0.0f : 1.0f / zz;
  if (tid < D) {
    float x = 0.0f;
#pragma unroll
    for (int w = 0; w < kPagedWaves; ++w) x += so[w][tid] * f[w];
    static_cast<uint16_t*>(a.O)[((long long)b * a.Hq + hq) * D + tid] = (uint16_t)float_to_bits<TYPE>(x * inv);
  }
  if (tid == 0 && a.lse)
    a.lse[(long long)b * a.Hq + hq] = zz == 0.0f ? -__builtin_huge_valf() : 0.69314718056f * (mm + __builtin_amdgcn_logf(zz));
}

}  // namespace

hipError_t launch_paged_decode(const PagedDecodeArgs& a, int d, int type, int format, hipStream_t stream) {
  return for_paged_types(d, type, format, [&](auto D, auto T, auto F) {
    hipLaunchKernelGGL((paged_decode_kernel<D(), T(), F()>), dim3(a.Hq, a.pool.B), dim3(kPagedWaves * kWave), 0, stream, a);
    return hipGetLastError();
  });
}

}  // namespace tilemix
