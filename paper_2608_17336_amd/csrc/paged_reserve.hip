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

// Sums over the threads before each one into before[i][], the sum over all into before[i][THREADS].
template <int THREADS, int N>
__device__ __forceinline__ void block_scan(const int (&x)[N], int (*before)[THREADS + 1], int (*waves)[THREADS / kWave]) {
  const int tid = threadIdx.x, wave = tid / kWave;
  int sum[N], base[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    sum[i] = wave_scan_most(x[i]);
    base[i] = 0;
    if (tid % kWave == kWave - 1) waves[i][wave] = sum[i];
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < THREADS / kWave - 1; ++w)   // (all are read: the reads then do not wait for one another)
#pragma unroll
    for (int i = 0; i < N; ++i) base[i] = add(base[i], w < wave ? waves[i][w] : 0);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    before[i][tid + 1] = add(base[i], sum[i]);
    if (tid == 0) before[i][0] = 0;
  }
  __syncthreads();
}

// What one sequence asks for.
struct Ask {
  int from, to;                 // lengths now and wanted
  int held, keep;               // first entry that it holds, and that it will hold if it grows
  bool fits;
  int need;                     // pages
  Ask() = default;
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
  Share() = default;
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
  // Sums of the runs of the threads before each one: pages needed; entries set, pages given back, new rows.
  enum { kEntries, kGives, kRowsSum };
  __shared__ int needed[1][THREADS + 1], sums[3][THREADS + 1], waves[3][THREADS / kWave];
  __shared__ int refused, taken, last;
  __shared__ Ask asks[THREADS];   // where a run is one sequence: looked up again and again
  const int tid = threadIdx.x, W = gridDim.x, wg = blockIdx.x, N = a.capacity;
  const int per = (a.B + THREADS - 1) / THREADS, b0 = min(tid * per, a.B), b1 = min(b0 + per, a.B);
  const int count = min(max(a.state[1], 0), N), head = (int)((uint32_t)max(a.state[0], 0) % (uint32_t)N);
  const int* needs = needed[0];
  auto ask = [&](int b) { return per == 1 ? asks[b] : Ask(a, b); };
  if (tid == 0) refused = taken = 0;
  int need[1] = {0};
  for (int b = b0; b < b1; ++b) {
    const Ask q(a, b);
    if (per == 1) asks[b] = q;
    need[0] = add(need[0], q.need);
  }
  block_scan<THREADS>(need, needed, waves);
  int own[3] = {0, 0, 0}, no = 0, take = 0, sum = needs[tid];
  for (int b = b0; b < b1; ++b) {
    const Ask q = ask(b);
    sum = add(sum, q.need);
    const Share s(a, q, sum, count);
    own[kEntries] = add(own[kEntries], s.entries);
    own[kGives] = add(own[kGives], s.give);
    own[kRowsSum] = add(own[kRowsSum], s.rows);
    if (s.entries) take += q.need;   // (not more than the list has)
    no += !q.fits || (q.need > 0 && sum > count);
  }
  __syncthreads();   // `waves` is used again
  if (no) atomicAdd(&refused, no);
  if (take) atomicAdd(&taken, take);
  block_scan<THREADS>(own, sums, waves);
  const int entries = sums[kEntries][THREADS], gives = sums[kGives][THREADS], rows = sums[kRowsSum][THREADS];

  auto ring = [&](int i) { return i < N ? i : i - N; };   // i < 2 N
  // All items in one line, so that a thread has few to wait for one after the other: entries, pages given back, rows.
  // (One copy of the search for the three of them: code that is read for the first time in a launch is waited for, too.
  // Four adjacent rows for a thread and one search took 12.8 us where this took 8.9, 410000 rows of 256 sequences.)
  const long long items = (long long)entries + gives + a.total;
  for (long long item = (long long)wg * THREADS + tid; item < items; item += (long long)W * THREADS) {
    const int kind = item < entries ? kEntries : item < (long long)entries + gives ? kGives : kRowsSum;
    const int k = kind == kEntries ? (int)item : kind == kGives ? (int)(item - entries) : (int)(item - entries - gives);
    int pos = -1, page = -1;
    if (kind != kRowsSum || k < rows) {
      // Whose item k is: the last thread with sums[kind][t] <= k, then its sequences.
      int t = 0;
#pragma unroll
      for (int step = THREADS / 2; step; step /= 2) t += sums[kind][t + step] <= k ? step : 0;
      int at = sums[kind][t], wanted = needs[t], below = 0, b = t * per;
      Ask q;
      Share s;
      for (;; ++b) {   // (k is less than the sum over all: its sequence comes before the run ends)
        q = ask(b);
        below = wanted;
        wanted = add(wanted, q.need);
        s = Share(a, q, wanted, count);
        const int n = kind == kEntries ? s.entries : kind == kGives ? s.give : s.rows;
        if (k - at < n || b + 1 >= min(t * per + per, a.B)) break;
        at += n;
      }
      const int i = k - at;
      pos = q.from + i;
      const int e = kind == kEntries ? s.e0 + i : kind == kGives ? s.g0 + i : pos >> a.page_shift;
      int* entry = a.table + b * a.stride_table + e;
      if (kind == kGives) {
        page = *entry;
        if (k < N - count) a.ids[ring(head + count + k)] = page;
        *entry = -1;
      } else if (kind == kEntries || a.slots) {   // (what the window leaves at once has no page)
        page = e < q.keep ? -1 : e < Ask::have(a, q.from) ? *entry : a.ids[ring(head + below + (e - q.first(a)))];
        if (kind == kEntries) *entry = page;
      }
    }
    if (kind == kRowsSum) {
      if (a.positions) a.positions[k] = pos;
      if (a.slots) a.slots[k] = page < 0 ? -1 : ((long long)page << a.page_shift) + (pos & ((1 << a.page_shift) - 1));
    }
  }
  if (a.in_place) {
    __syncthreads();   // all of the workgroup's reads are done
    if (tid == 0) last = W == 1 || atomicInc(reinterpret_cast<unsigned*>(a.state + 3), W - 1) == (unsigned)W - 1;
    __syncthreads();
  }
  if (a.in_place ? !last : wg != 0) return;
  int wanted = needs[tid], at = sums[kRowsSum][tid];
  for (int b = b0; b < b1; ++b) {
    const Ask q = ask(b);
    wanted = add(wanted, q.need);
    const Share s(a, q, wanted, count);
    if (a.cu) a.cu[b] = at;
    at = add(at, s.rows);
    a.lens_out[b] = s.len;
    if (a.window > 0) a.first_held[b] = s.held;
  }
  if (tid == 0) {
    if (a.cu) a.cu[a.B] = rows;
    a.state_out[0] = ring(head + taken);
    a.state_out[1] = count - taken + min(gives, N - count);
    a.state_out[2] = refused;
    a.state_out[3] = 0;
  }
}

}  // namespace

hipError_t launch_paged_reserve(ReserveArgs a, hipStream_t stream) {
  if (!a.positions && !a.slots) a.total = 0;
  // (first_held always is; other overlaps are refused.)
  a.in_place = a.window > 0 || a.lens_out == a.old_lens || a.lens_out == a.want || a.state_out == a.state;
  // (How many entries change is not known here: a part of those that could.)  Workgroups that write the state in place count
  // themselves one after the other, some 10 ns each: fewer and larger ones.
  const long long items = a.total + std::min<long long>((long long)a.B * a.max_pages, a.capacity) / 8;
  const bool large = a.B > 256 || (a.in_place && items > 32768);
  const unsigned threads = large ? 1024 : 256;
  const unsigned grid = (unsigned)std::min<long long>(a.in_place ? 128 : 512, std::max<long long>(1, items / threads));
  if (large) hipLaunchKernelGGL((paged_reserve_kernel<1024>), dim3(grid), dim3(1024), 0, stream, a);
  else hipLaunchKernelGGL((paged_reserve_kernel<256>), dim3(grid), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace tilemix
