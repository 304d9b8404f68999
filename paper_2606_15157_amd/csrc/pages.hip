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
// write8_kernel: the same in 8 bits.  A row's largest value is found by its 16 lanes, its codes are the hardware's rounding of values that a
//   power of two has scaled, which is exact; 16371 rows of 8 heads in 21.5 us (101 MB, 4.7 TB/s).
// read_kernel, read8_kernel: the way back; four prompts of 8192 rows of 8 heads from 8 bits in 37.5 us back to back (202 MB, 5.4 TB/s).
#include <hip/hip_runtime.h>

#include "paged.h"

namespace rkv {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

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

// Where a (token, head) row of a call lies among the rows and in the pool.
struct RowPlace {
  int o, t, h, page, at;
  bool there;      // whether its slot is one of the pool's
};
__device__ __forceinline__ RowPlace place_of(const WriteLaunch& W, int item) {
  RowPlace x;
  const int row = div_by(item, W.by_head), slot = W.r.slots[row];
  x.h = item - row * W.p.n_kv_heads;
  x.o = div_by(row, W.by_token);
  x.t = row - x.o * W.r.n_tokens;
  x.there = (uint32_t)slot < (uint32_t)W.n_slots;
  x.page = div_by(x.there ? slot : 0, W.by_page);
  x.at = slot - x.page * W.p.page_size;
  return x;
}
// blockIdx.x: 16 (token, head) rows, 16 lanes each.
__device__ __forceinline__ int item_of() { return blockIdx.x * 16 + (threadIdx.x >> 4); }
// This lane's eight values of a row, among the rows and in a pool of 16-bit rows; its eight codes; the row's exponent.
__device__ __forceinline__ u32x4* k_row(const WriteLaunch& W, const RowPlace& x) {
  return reinterpret_cast<u32x4*>((uint16_t*)W.r.k + x.o * W.r.k_outer + x.t * W.r.k_token + x.h * W.r.k_head) + (threadIdx.x & 15);
}
__device__ __forceinline__ u32x4* v_row(const WriteLaunch& W, const RowPlace& x) {
  return reinterpret_cast<u32x4*>((uint16_t*)W.r.v + x.o * W.r.v_outer + x.t * W.r.v_token + x.h * W.r.v_head) + (threadIdx.x & 15);
}
__device__ __forceinline__ u32x4* k_slot(const WriteLaunch& W, const RowPlace& x) {
  return reinterpret_cast<u32x4*>(static_cast<uint16_t*>(W.p.k) + x.page * W.p.k_page + x.at * W.p.k_slot + x.h * W.p.k_head) + (threadIdx.x & 15);
}
__device__ __forceinline__ u32x4* v_slot(const WriteLaunch& W, const RowPlace& x) {
  return reinterpret_cast<u32x4*>(static_cast<uint16_t*>(W.p.v) + x.page * W.p.v_page + x.at * W.p.v_slot + x.h * W.p.v_head) + (threadIdx.x & 15);
}
__device__ __forceinline__ u32x2* k_codes(const WriteLaunch& W, const RowPlace& x) {
  return reinterpret_cast<u32x2*>(static_cast<uint8_t*>(W.p.k) + x.page * W.p.k_page + x.at * W.p.k_slot + x.h * W.p.k_head) + (threadIdx.x & 15);
}
__device__ __forceinline__ u32x2* v_codes(const WriteLaunch& W, const RowPlace& x) {
  return reinterpret_cast<u32x2*>(static_cast<uint8_t*>(W.p.v) + x.page * W.p.v_page + x.at * W.p.v_slot + x.h * W.p.v_head) + (threadIdx.x & 15);
}
__device__ __forceinline__ uint8_t* scale_at(const Scales& s, const RowPlace& x) { return s.at + x.page * s.page + x.h * s.head + x.at * s.slot; }

__global__ __launch_bounds__(256) void write_kernel(const WriteLaunch W) {
  if (item_of() >= W.n_items) return;
  const RowPlace x = place_of(W, item_of());
  if (!x.there) return;
  const u32x4 k = *k_row(W, x), v = *v_row(W, x);
  *k_slot(W, x) = k;
  *v_slot(W, x) = v;
}

// A row of 128 values as e4m3 codes and a power of two 2^e, e the least with max |x| <= 448 2^e among those that leave every code
// times 2^e a value of the row's own type (bf16 -117 .. 120, fp16 -15 .. 8, and at the largest e codes to 240): x 2^-e is exact, the
// code its one rounding, and what is read back is exact again.  What is not finite has no part in e, and NaN for a code.
// Returns this lane's eight codes; byte: e + 127.
template <bool kF16>
__device__ __forceinline__ u32x2 encode(u32x4 v, uint32_t& byte) {
  constexpr uint32_t kLeast = kF16 ? 112 : 10, kMost = kF16 ? 135 : 247;
  constexpr uint32_t kInf = 0x7f800000u;
  float x[8];
  uint32_t top = 0;     // bits of non-negative floats are in their order
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t half = i & 1 ? v[i >> 1] >> 16 : v[i >> 1] & 0xffffu;
    if constexpr (kF16) x[i] = (float)__builtin_bit_cast(_Float16, (uint16_t)half);
    else x[i] = __uint_as_float(half << 16);
    const uint32_t a = __float_as_uint(x[i]) & 0x7fffffffu;
    top = max(top, a < kInf ? a : 0u);
  }
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
  // floor(log2 top) - 8, one more if top exceeds 1.75 of its power of two: that carries into the exponent
  const int e = (int)((top + 0x1fffffu) >> 23) - 8;
  byte = (uint32_t)min(max(e, (int)kLeast), (int)kMost);
  const float down = __uint_as_float((254u - byte) << 23), most = byte == kMost ? 240.f : 448.f;
  u32x2 code;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    float y[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float z = x[4 * i + j];
      y[j] = (__float_as_uint(z) & 0x7fffffffu) < kInf ? fminf(fmaxf(z * down, -most), most) : __builtin_nanf("");
    }
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    code[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
  }
  return code;
}
template <bool kF16>
__global__ __launch_bounds__(256) void write8_kernel(const WriteLaunch W) {
  if (item_of() >= W.n_items) return;      // by whole rows: their 16 lanes stay together
  const RowPlace x = place_of(W, item_of());
  if (!x.there) return;
  const u32x4 k = *k_row(W, x), v = *v_row(W, x);
  uint32_t k_byte, v_byte;
  const u32x2 kc = encode<kF16>(k, k_byte), vc = encode<kF16>(v, v_byte);
  *k_codes(W, x) = kc;
  *v_codes(W, x) = vc;
  if ((threadIdx.x & 15) == 0) {
    *scale_at(W.ks, x) = (uint8_t)k_byte;
    *scale_at(W.vs, x) = (uint8_t)v_byte;
  }
}

// Rows read back; kPast: more than the L2 caches hold go past them (four prompts of 8192, 134 MB: 46 us a call -> 39).
constexpr int64_t kPastBytes = int64_t(32) << 20;
template <bool kPast>
__device__ __forceinline__ void store_rows(const WriteLaunch& W, const RowPlace& x, u32x4 k, u32x4 v) {
  if constexpr (kPast) {
    __builtin_nontemporal_store(k, k_row(W, x));
    __builtin_nontemporal_store(v, v_row(W, x));
  } else {
    *k_row(W, x) = k;
    *v_row(W, x) = v;
  }
}
template <bool kPast>
__global__ __launch_bounds__(256) void read_kernel(const WriteLaunch W) {
  if (item_of() >= W.n_items) return;
  const RowPlace x = place_of(W, item_of());
  u32x4 k = {0, 0, 0, 0}, v = k;
  if (x.there) {
    k = *k_slot(W, x);
    v = *v_slot(W, x);
  }
  store_rows<kPast>(W, x, k, v);
}

template <bool kF16>
__device__ __forceinline__ u32x4 decode(u32x2 code, uint32_t byte) {
  const float scale = __uint_as_float(byte << 23);
  u32x4 x;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t c = code[i >> 1];
    if constexpr (kF16)
      x[i] = __builtin_bit_cast(uint32_t, i & 1 ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c, scale, true) : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c, scale, false));
    else
      x[i] = __builtin_bit_cast(uint32_t, i & 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, scale, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, scale, false));
  }
  return x;
}
template <bool kF16, bool kPast>
__global__ __launch_bounds__(256) void read8_kernel(const WriteLaunch W) {
  if (item_of() >= W.n_items) return;
  const RowPlace x = place_of(W, item_of());
  u32x4 k = {0, 0, 0, 0}, v = k;
  if (x.there) {
    const u32x2 kc = *k_codes(W, x), vc = *v_codes(W, x);
    const uint32_t k_byte = *scale_at(W.ks, x), v_byte = *scale_at(W.vs, x);
    k = decode<kF16>(kc, k_byte);
    v = decode<kF16>(vc, v_byte);
  }
  store_rows<kPast>(W, x, k, v);
}

}  // namespace

int launch_resize(const ResizeLaunch& R, void* stream) {
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  const bool fill = R.r.max_new <= kResizeSlots;
  resize_kernel<<<1, kResizeThreads, 0, st>>>(R, fill);
  if (!fill) slots_kernel<<<(unsigned)(((int64_t)R.r.max_new + 255) / 256), 256, 0, st>>>(R);
  return (int)hipGetLastError();
}

namespace {
using RowsKernel = void(const WriteLaunch);
int launch_items(RowsKernel* kernel, const WriteLaunch& W, void* stream) {
  kernel<<<(unsigned)(((int64_t)W.n_items + 15) / 16), 256, 0, reinterpret_cast<hipStream_t>(stream)>>>(W);
  return (int)hipGetLastError();
}
}  // namespace

int launch_write(const WriteLaunch& W, void* stream) { return launch_items(write_kernel, W, stream); }
int launch_write8(const WriteLaunch& W, void* stream) {
  return launch_items(W.p.dtype == RKV_F16 ? write8_kernel<true> : write8_kernel<false>, W, stream);
}
int launch_read(const WriteLaunch& W, void* stream) {
  const bool past = (int64_t)W.n_items * 4 * kHeadDim > kPastBytes;
  return launch_items(past ? read_kernel<true> : read_kernel<false>, W, stream);
}
int launch_read8(const WriteLaunch& W, void* stream) {
  const bool past = (int64_t)W.n_items * 4 * kHeadDim > kPastBytes;
  if (W.p.dtype == RKV_F16) return launch_items(past ? read8_kernel<true, true> : read8_kernel<true, false>, W, stream);
  return launch_items(past ? read8_kernel<false, true> : read8_kernel<false, false>, W, stream);
}

}  // namespace rkv
