// paged_reserve.hip -- pages for new tokens: page tables, positions and slots from request lengths (latency-bound).
//
// One launch.  Every workgroup goes over all lengths by itself: a thread takes a run of sequences, and three block-wide
// prefix sums (pages wanted; entries taken, pages given back and new rows of the sequences served) say where each run's
// shares begin.  Then the workgroups share the entries and rows, which look their sequence up in those sums.  The
// lengths and the list's state may be written over their old values: the last workgroup to arrive does that, when all
// others have read what they need.
#include "tilemix_device.h"
#include "tilemix_internal.h"

#include <algorithm>

namespace tilemix {

namespace {

// Sums stop here: beyond the largest list, so that what is larger is more than any list has.
constexpr int kMost = (1 << 30) - 1;
__device__ __forceinline__ int add(int x, int y) { return min(x + y, kMost); }   // x, y <= kMost

__device__ __forceinline__ int wave_scan_most(int x) {
  x = add(x, dpp<0x111>(0, x));
  x = add(x, dpp<0x112>(0, x));
  x = add(x, dpp<0x114>(0, x));
  x = add(x, dpp<0x118>(0, x));
  x = add(x, dpp<0x142, 0xa>(0, x));
  x = add(x, dpp<0x143, 0xc>(0, x));
  return x;
}

// Sums over the threads before each one into before[], before[THREADS] the sum over all.
template <int THREADS>
__device__ __forceinline__ void block_scan(int x, int* before, int* waves) {
  const int tid = threadIdx.x, wave = tid / kWave;
  const int sum = wave_scan_most(x);
  if (tid % kWave == kWave - 1) waves[wave] = sum;
  __syncthreads();
  int base = 0;
  for (int w = 0; w < wave; ++w) base = add(base, waves[w]);
  before[tid + 1] = add(base, sum);
  if (tid == 0) before[0] = 0;
  __syncthreads();
}

// What one sequence asks for.
struct Ask {
  int from, to;                 // lengths now and wanted
  int held, keep;               // first entry that it holds, and that it will hold if it grows
  bool fits;
  int need;                     // pages
  __device__ __forceinline__ Ask(const ReserveArgs& a, int b) {
    const long long cap = (long long)a.max_pages << a.page_shift;
    from = (int)min((long long)max(a.old_lens[b], 0), cap);
    to = max(a.want[b], 0);
    fits = to <= cap;
    held = keep = 0;
    if (a.window > 0) {
      held = min(max(a.first_held[b], 0), have(a, from));
      keep = max(held, (int)(max((long long)to - a.window, 0ll) >> a.page_shift));
    }
    need = fits && to > from ? max(0, have(a, to) - first(a)) : 0;
  }
  __device__ __forceinline__ static int have(const ReserveArgs& a, int len) {
    return (int)(((long long)len + (1 << a.page_shift) - 1) >> a.page_shift);
  }
  // First entry that takes a page.
  __device__ __forceinline__ int first(const ReserveArgs& a) const { return max(have(a, from), keep); }
};

// What it gets.  Entries e0 .. e0 + entries - 1 are set (those in front of `first` to -1), pages of g0 .. g0 + give - 1
// go back.
struct Share {
  int len, held, rows = 0, e0 = 0, entries = 0, g0 = 0, give = 0;
  // sum: pages wanted by it and all before it.
  __device__ __forceinline__ Share(const ReserveArgs& a, const Ask& q, int sum, int count) {
    const bool ok = q.fits && (q.need == 0 || sum <= count);
    len = ok ? q.to : q.from;
    held = q.held;
    if (!ok) return;
    const int have = Ask::have(a, q.from);
    if (q.to > q.from) {
      held = q.keep;
      rows = q.to - q.from;
      e0 = have;
      entries = Ask::have(a, q.to) - have;
      g0 = q.held;
      give = min(q.keep, have) - g0;
    } else {
      held = min(q.held, Ask::have(a, q.to));
      g0 = max(Ask::have(a, q.to), q.held);
      give = have - g0;
    }
  }
};

template <int THREADS>
__global__ __launch_bounds__(THREADS) void paged_reserve_kernel(ReserveArgs a) {
  // Sums of the runs of the threads before each one.
  __shared__ int needs[THREADS + 1], entries[THREADS + 1], gives[THREADS + 1], rows[THREADS + 1];
  __shared__ int waves[4][THREADS / kWave];
  __shared__ int refused, taken, last;
  const int tid = threadIdx.x, W = gridDim.x, wg = blockIdx.x, N = a.capacity;
  const int per = (a.B + THREADS - 1) / THREADS, b0 = min(tid * per, a.B), b1 = min(b0 + per, a.B);
  const int count = min(max(a.state[1], 0), N), head = (int)((uint32_t)max(a.state[0], 0) % (uint32_t)N);
  if (tid == 0) refused = taken = 0;
  int need = 0;
  for (int b = b0; b < b1; ++b) need = add(need, Ask(a, b).need);
  block_scan<THREADS>(need, needs, waves[0]);
  int set = 0, give = 0, row = 0, no = 0, take = 0, sum = needs[tid];
  for (int b = b0; b < b1; ++b) {
    const Ask q(a, b);
    sum = add(sum, q.need);
    const Share s(a, q, sum, count);
    set = add(set, s.entries);
    give = add(give, s.give);
    row = add(row, s.rows);
    if (s.entries) take += q.need;   // (not more than the list has)
    no += !q.fits || (q.need > 0 && sum > count);
  }
  block_scan<THREADS>(set, entries, waves[1]);
  block_scan<THREADS>(give, gives, waves[2]);
  block_scan<THREADS>(row, rows, waves[3]);
  if (no) atomicAdd(&refused, no);
  if (take) atomicAdd(&taken, take);

  // f(sequence, Ask, Share, item within its share, pages wanted before it) of item k, which `before` counts.
  auto find = [&](const int* before, int k, auto&& part, auto&& f) {
    int t = 0;   // the last thread with before[t] <= k
#pragma unroll
    for (int step = THREADS / 2; step; step /= 2) t += before[t + step] <= k ? step : 0;
    int at = before[t], wanted = needs[t];
    for (int b = t * per; b < min(t * per + per, a.B); ++b) {
      const Ask q(a, b);
      const int below = wanted;
      wanted = add(wanted, q.need);
      const Share s(a, q, wanted, count);
      const int n = part(s);
      if (k - at < n) {
        f(b, q, s, k - at, below);
        return;
      }
      at += n;
    }
  };
  auto ring = [&](int i) { return i < N ? i : i - N; };   // i < 2 N
  const int stride = W * THREADS, at0 = wg * THREADS + tid;
  for (int k = at0; k < entries[THREADS]; k += stride)
    find(entries, k, [](const Share& s) { return s.entries; }, [&](int b, const Ask& q, const Share& s, int i, int below) {
      const int e = s.e0 + i, n = e - q.first(a);
      a.table[b * a.stride_table + e] = n >= 0 ? a.ids[ring(head + below + n)] : -1;
    });
  for (int k = at0; k < gives[THREADS]; k += stride)
    find(gives, k, [](const Share& s) { return s.give; }, [&](int b, const Ask&, const Share& s, int i, int) {
      int* entry = a.table + b * a.stride_table + s.g0 + i;
      if (k < N - count) a.ids[ring(head + count + k)] = *entry;
      *entry = -1;
    });
  if (a.positions || a.slots) {
    for (int k = at0; k < a.total; k += stride) {
      int pos = -1;
      long long slot = -1;
      if (k < rows[THREADS])
        find(rows, k, [](const Share& s) { return s.rows; }, [&](int b, const Ask& q, const Share&, int i, int below) {
          pos = q.from + i;
          const int e = pos >> a.page_shift;
          if (!a.slots || e < q.keep) return;   // (the window leaves it at once: it has no page)
          const int page = e < Ask::have(a, q.from) ? a.table[b * a.stride_table + e]
                                                    : a.ids[ring(head + below + (e - q.first(a)))];
          if (page >= 0) slot = ((long long)page << a.page_shift) + (pos & ((1 << a.page_shift) - 1));
        });
      if (a.positions) a.positions[k] = pos;
      if (a.slots) a.slots[k] = slot;
    }
  }
  if (a.cu && wg == 0) {
    int at = rows[tid], wanted = needs[tid];
    for (int b = b0; b < b1; ++b) {
      const Ask q(a, b);
      wanted = add(wanted, q.need);
      a.cu[b] = at;
      at = add(at, Share(a, q, wanted, count).rows);
    }
    if (tid == 0) a.cu[a.B] = rows[THREADS];
  }
  __syncthreads();   // all of the workgroup's reads are done
  if (tid == 0) last = W == 1 || atomicInc(reinterpret_cast<unsigned*>(a.state + 3), W - 1) == (unsigned)W - 1;
  __syncthreads();
  if (!last) return;
  int wanted = needs[tid];
  for (int b = b0; b < b1; ++b) {
    const Ask q(a, b);
    wanted = add(wanted, q.need);
    const Share s(a, q, wanted, count);
    a.lens_out[b] = s.len;
    if (a.window > 0) a.first_held[b] = s.held;
  }
  if (tid == 0) {
    a.state_out[0] = ring(head + taken);
    a.state_out[1] = min(count - taken + min(gives[THREADS], N - count), N);
    a.state_out[2] = refused;
    a.state_out[3] = 0;
  }
}

}  // namespace

hipError_t launch_paged_reserve(const ReserveArgs& a, hipStream_t stream) {
  const bool many = a.B > 256;
  const int threads = many ? 1024 : 256;
  const long long items = std::max<long long>(a.positions || a.slots ? a.total : 0,
                                              std::min<long long>((long long)a.B * a.max_pages, a.capacity) / 4);
  const unsigned grid = (unsigned)std::min<long long>(256, std::max<long long>(1, items / (4 * threads)));
  if (many) hipLaunchKernelGGL((paged_reserve_kernel<1024>), dim3(grid), dim3(1024), 0, stream, a);
  else hipLaunchKernelGGL((paged_reserve_kernel<256>), dim3(grid), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace tilemix
