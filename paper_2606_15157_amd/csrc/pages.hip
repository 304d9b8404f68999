// Paged caches for gfx950: block tables and slot maps from request lengths, and new rows to their slots.
//
// resize_kernel: one workgroup.  A scheduler's turn is a few hundred lengths and, with a decode step, a handful of
//   pages: latency, not bandwidth.  The three prefix sums (pages taken, pages given back, new tokens) need every
//   sequence before any page moves, so one workgroup scans them once and keeps them in LDS, where each page and each
//   new token finds its sequence by bisection: the work is spread by pages and tokens, not by sequences.  5.1 us for 64
//   sequences that get a token each, 9.8 us for 192 of which 40 enter with up to 32K tokens and 48 end (four lookups of a thread
//   side by side: 11.0).
// slots_kernel: the slot map of many new tokens (entering prompts), over the whole chip, from the tables as written.
// write_kernel: 16 lanes a row, 16 bytes each of K and of V; bound by HBM: 16371 rows of 8 heads in 21.6 us (134 MB), 28 us
//   back to back (4.8 TB/s, what a large copy reaches).
#include <hip/hip_runtime.h>

#include "paged.h"

namespace rkv {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kResizeThreads = 1024;
constexpr int kResizeSlots = 8192;      // slots the workgroup fills itself

__device__ __forceinline__ int div_by(int n, FastDiv d) { return (int)(__umulhi((uint32_t)n << 1, d.mul) >> d.shift); }

// ceil(n / d), `by` made for d.
__device__ __forceinline__ int pages_of(int n, FastDiv by, int d) {
  const int q = div_by(n, by);
  return q + (n != q * d);
}
// (a + j) mod n for a, j < n.
__device__ __forceinline__ uint32_t wrap(uint32_t a, uint32_t j, uint32_t n) {
  const uint32_t x = a + j;
  return x >= n ? x - n : x;
}

// Last s of [0, n) with start[s] <= j (start ascending, start[0] <= j).
__device__ __forceinline__ int owner(const int32_t* start, int n, int j) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (start[mid] <= j) lo = mid;
    else hi = mid;
  }
  return lo;
}

// The flat slot of new token j, with `start` the sequences' first new tokens; -1 for a page outside the pool.
__device__ __forceinline__ int slot_of(const ResizeLaunch& R, const int32_t* start, int j) {
  const rkv_resize& r = R.r;
  const int s = owner(start, r.n_seqs, j);
  const int at = r.new_lens[s] - (start[s + 1] - j);
  const int col = div_by(at, R.by_page);
  const int page = r.table[s * r.table_stride + col];
  return (uint32_t)page < (uint32_t)r.n_pages ? page * r.page_size + at - col * r.page_size : -1;
}

__global__ __launch_bounds__(kResizeThreads) void resize_kernel(const ResizeLaunch R, const bool fill) {
  __shared__ int32_t sTake[kResizeMaxSeqs + 1], sGive[kResizeMaxSeqs + 1], sAdd[kResizeMaxSeqs + 1];
  __shared__ int64_t sWave[3][kResizeThreads / 64];
  const rkv_resize& r = R.r;
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  const int n = r.n_seqs, page = r.page_size, cap = r.n_pages;
  const int per = (n + kResizeThreads - 1) / kResizeThreads;     // consecutive sequences of a thread
  const int s0 = min(n, tid * per), s1 = min(n, s0 + per);
  const int head = r.cursor[0], count = r.cursor[1];
  const int64_t most = (int64_t)r.max_pages * page;
  // totals in 64 bits: lengths are not yet known to be sound
  int64_t sum[3] = {0, 0, 0};
  int bad = (uint32_t)head >= (uint32_t)cap || (uint32_t)count > (uint32_t)cap;
  for (int s = s0; s < s1; ++s) {
    const int a = r.lens[s], b = r.new_lens[s];
    if (a < 0 || b < 0 || a > most || b > most) {
      bad = 1;
      continue;
    }
    const int have = pages_of(a, R.by_page, page), want = pages_of(b, R.by_page, page);
    sum[0] += max(0, want - have);
    sum[1] += max(0, have - want);
    sum[2] += max(0, b - a);
  }
  int64_t before[3], total[3];
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    int64_t x = sum[k];
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int64_t y = __shfl_up((long long)x, o);
      if (lane >= o) x += y;
    }
    before[k] = x - sum[k];
    if (lane == 63) sWave[k][wv] = x;
  }
  bad = __syncthreads_or(bad);
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    total[k] = 0;
#pragma unroll
    for (int i = 0; i < kResizeThreads / 64; ++i) {
      if (i == wv) before[k] += total[k];
      total[k] += sWave[k][i];
    }
  }
  uint32_t status = 0;
  if (bad || total[2] > r.max_new || (total[0] <= count && count - total[0] + total[1] > cap)) status = RKV_PAGES_INVALID;
  else if (total[0] > count) status = RKV_PAGES_EXHAUSTED;
  if (tid == 0) {
    *r.status = status;
    r.cursor_out[0] = status ? head : (int)wrap(head, (uint32_t)total[0], cap);
    r.cursor_out[1] = status ? count : (int)(count - total[0] + total[1]);
  }
  if (status) {
    for (int s = s0; s < s1; ++s) r.lens_out[s] = r.lens[s];
    for (int s = tid; s <= n; s += kResizeThreads) r.cu_new[s] = 0;
    if (fill)
      for (int j = tid; j < r.max_new; j += kResizeThreads) r.slots[j] = -1;
    return;
  }
  int take = (int)before[0], give = (int)before[1], add = (int)before[2];
  for (int s = s0; s < s1; ++s) {
    const int a = r.lens[s], b = r.new_lens[s];
    const int have = pages_of(a, R.by_page, page), want = pages_of(b, R.by_page, page);
    sTake[s] = take;
    sGive[s] = give;
    sAdd[s] = add;
    r.cu_new[s] = add;
    r.lens_out[s] = b;
    take += max(0, want - have);
    give += max(0, have - want);
    add += max(0, b - a);
  }
  if (tid == 0) {
    sTake[n] = (int)total[0];
    sGive[n] = (int)total[1];
    sAdd[n] = (int)total[2];
    r.cu_new[n] = (int)total[2];
  }
  __syncthreads();
  for (int64_t i = tid; i < total[0]; i += kResizeThreads) {
    const int j = (int)i, s = owner(sTake, n, j), b = r.new_lens[s];
    const int want = pages_of(b, R.by_page, page);
    r.table[s * r.table_stride + want - (sTake[s + 1] - j)] = r.ring[wrap(head, j, cap)];
  }
  __syncthreads();   // pages given back may reach round to ring entries just taken
  const uint32_t tail = wrap(head, count, cap);   // total[1] <= cap: it leaves at most cap pages free
  for (int64_t i = tid; i < total[1]; i += kResizeThreads) {
    const int j = (int)i, s = owner(sGive, n, j), b = r.new_lens[s];
    const int want = pages_of(b, R.by_page, page);
    r.ring[wrap(tail, j, cap)] = r.table[s * r.table_stride + want + j - sGive[s]];
  }
  if (fill)
    for (int j = tid; j < r.max_new; j += kResizeThreads) r.slots[j] = j < (int)total[2] ? slot_of(R, sAdd, j) : -1;
}

__global__ __launch_bounds__(256) void slots_kernel(const ResizeLaunch R) {
  const rkv_resize& r = R.r;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= r.max_new) return;
  const int j = (int)i;
  r.slots[j] = j < r.cu_new[r.n_seqs] ? slot_of(R, r.cu_new, j) : -1;
}

// blockIdx.x: 16 (token, head) rows, 16 lanes each.
__global__ __launch_bounds__(256) void write_kernel(const WriteLaunch W) {
  const int item = blockIdx.x * 16 + (threadIdx.x >> 4), c = 8 * (threadIdx.x & 15);
  if (item >= W.n_items) return;
  const rkv_rows& r = W.r;
  const rkv_pages& p = W.p;
  const int row = div_by(item, W.by_head), h = item - row * p.n_kv_heads;
  const int slot = r.slots[row];
  if ((uint32_t)slot >= (uint32_t)W.n_slots) return;
  const int o = div_by(row, W.by_token), t = row - o * r.n_tokens;
  const int page = div_by(slot, W.by_page), at = slot - page * p.page_size;
  const u32x4 k = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(r.k) + o * r.k_outer + t * r.k_token + h * r.k_head + c);
  const u32x4 v = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(r.v) + o * r.v_outer + t * r.v_token + h * r.v_head + c);
  *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(p.k) + page * p.k_page + at * p.k_slot + h * p.k_head + c) = k;
  *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(p.v) + page * p.v_page + at * p.v_slot + h * p.v_head + c) = v;
}

}  // namespace

int launch_resize(const ResizeLaunch& R, void* stream) {
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  const bool fill = R.r.max_new <= kResizeSlots;
  resize_kernel<<<1, kResizeThreads, 0, st>>>(R, fill);
  if (!fill) slots_kernel<<<(unsigned)(((int64_t)R.r.max_new + 255) / 256), 256, 0, st>>>(R);
  return (int)hipGetLastError();
}

int launch_write(const WriteLaunch& W, void* stream) {
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  write_kernel<<<(unsigned)(((int64_t)W.n_items + 15) / 16), 256, 0, st>>>(W);
  return (int)hipGetLastError();
}

}  // namespace rkv
