// Attention of new tokens over a paged cache for gfx950.
//
// Rows of one KV head are its G query heads' tokens, row = token G + g: the group shares every key it reads, and a short
// chunk fills a tile of rows.  A workgroup takes a tile of 128 rows of one sequence and KV head, 32 rows a wave, and
// streams the visible keys in tiles of 64 through LDS (DMA, two buffers).
//
//   S^T = K Q^T   32x32x16 MFMA, keys x rows: a lane holds 16 keys of one row (column lane % 32) per 32 keys, so the
//                 softmax statistics of a row are one value a lane, the two halves of a wave exchanged once a tile;
//   O^T += V^T P^T   the lane's own probabilities, rounded to 16 bits, are the B operand as they stand when the sum over
//                 keys runs in the order the lane holds them: slots 0-3 of a half are keys 4 half + 0..3, slots 4-7 keys
//                 8 + 4 half + 0..3 of each 16.  V^T in that order is two transposing LDS reads.  P never leaves registers.
//
// P in 16 bits is what the matrix instructions take at this rate; it takes the outputs' error against 64 bits from 1.6e-3 (an
// output's own rounding to bf16) to at most 1.9e-3, in fp16 from 2.1e-4 to 2.4e-4.
//
// One pass with a running maximum m (log2 units), sum l and output O^T per row, rescaled only when a maximum outgrows the
// reference by more than 8 (factors of exp2(8) at most in P, which has the exponent range for it: in fp16 the reference lies
// 2^7 below the maximum).
//
// Prompts are a workgroup per row tile and head.  Up to kListed tiles of long sequences (decode steps, chunks) are dealt out by
// key tiles: every workgroup adds up the same list of tiles' costs from cu_q and lens, which the host does not know, and
// takes an equal, consecutive share, however ragged the batch.  A share's first and last rows may be part of an item: those
// partial sums go to the workspace, and join_kernel adds them in the order of the keys.  Nothing depends on what an earlier
// call left there.  At most 16 rows (decode steps) go the narrow way below.
//
// Measured with 32 query and 8 KV heads, bf16, pages of 16: a prompt of 16384 1.95 ms (1.13 PFLOP/s; the matrix pipes are busy
// 59 % of the cycles, and the power limit sets the clock: fewer LDS reads or instructions count, not more overlap); 512
// tokens after 32768 287 us (0.97 PFLOP/s); 64 evicted caches of 1024 rows 41 us (6.5 TB/s of keys and values), 64 ragged
// sequences of 512 to 8192 159 us (5.1 TB/s), one token after 1024 12.0 us (16 key tiles one after another).
#include <hip/hip_runtime.h>

#include <type_traits>

#include "lds_dma.h"
#include "paged.h"

namespace rkv {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

constexpr int kRows = kAttendRows;         // rows of a workgroup, 32 a wave
constexpr int kKeys = 64;                  // keys of a streamed tile
constexpr int kShares = kAttendShares;
constexpr int kListed = kAttendListed;
constexpr int kAhead = 11;                 // of a tile's 16 pairs of probabilities, those computed between the products of K
constexpr int kTileBytes = kKeys * kHeadDim * 2;
constexpr int64_t kStrideEnd = int64_t(1) << 31;   // page strides (elements) whose bytes 32 bits hold
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kGrow = 8.f;               // log2 units a maximum may outgrow the reference by
// Log2 units of the reference below the maximum it was set at.  Probabilities then reach 2^(kGrow + kUnder): fp16 holds 65504, and
// with 2^7 a row's small ones keep half a step of 2^-32 of its largest.  With none, keys 17 nats below an attention sink
// were 0 in the output and not in its divisor.  bf16 has the range of the sums.
template <bool kF16>
constexpr float kUnder = kF16 ? 7.f : 0.f;

__device__ __align__(256) uint32_t zero_row[kHeadDim / 2];   // what a slot outside the visible ones reads as

__device__ __forceinline__ int div_by(int n, FastDiv d) { return (int)(__umulhi((uint32_t)n << 1, d.mul) >> d.shift); }

// Four DMA instructions of 16 bytes per lane, to LDS 1 KiB apart: [base + off[j] + 1024 j] -> lds_base + 1024 j (+ 16 lane); the instruction offsets
// apply to both addresses.
__device__ __forceinline__ void dma16s_four(const char* base, const uint32_t (&off)[4], uint32_t lds_base) {
  uint32_t saved;
  asm volatile(
      "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %6\n\ts_nop 0\n\t"
      "global_load_lds_dwordx4 %1, %5\n\t"
      "global_load_lds_dwordx4 %2, %5 offset:1024\n\t"
      "global_load_lds_dwordx4 %3, %5 offset:2048\n\t"
      "global_load_lds_dwordx4 %4, %5 offset:3072\n\ts_mov_b32 m0, %0"
      : "=&s"(saved)
      : "v"(off[0]), "v"(off[1]), "v"(off[2]), "v"(off[3]), "s"(base), "s"(lds_base)
      : "memory");
}

template <bool kF16>
__device__ __forceinline__ f32x16 mma32(u32x4 a, u32x4 b, f32x16 c) {
  if constexpr (kF16) return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
// 16 x 16, 32 and 16 deep.
template <bool kF16>
__device__ __forceinline__ f32x4 mma16(u32x4 a, u32x4 b, f32x4 c) {
  if constexpr (kF16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
template <bool kF16>
__device__ __forceinline__ f32x4 mma16s(u32x2 a, u32x2 b, f32x4 c) {
  if constexpr (kF16) return __builtin_amdgcn_mfma_f32_16x16x16f16(__builtin_bit_cast(f16x4, a), __builtin_bit_cast(f16x4, b), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4, a), __builtin_bit_cast(s16x4, b), c, 0, 0, 0);
}
// Two values rounded to nearest even.
template <bool kF16>
__device__ __forceinline__ uint32_t pack(float x, float y) {
  const f32x2 v = {x, y};
  if constexpr (kF16) return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2));
  else return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}
__device__ __forceinline__ u32x4 lds_read16(uint32_t at) { return *(const __attribute__((address_space(3))) u32x4*)(uintptr_t)at; }
__device__ __forceinline__ u32x2 lds_read_tr(uint32_t at) {
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(uintptr_t)at));
}
// log sum exp of a row from its sum and what that is relative to (log2 units).
__device__ __forceinline__ float row_lse(float m, float l) { return l == 0.f ? -__builtin_inff() : m / kLog2e + logf(l); }
// All of this wave's DMA is in and its LDS reads are done, then the workgroup's.
__device__ __forceinline__ void tile_sync() {
  wait_vmcnt<0>();
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt 0
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}
__device__ __forceinline__ float max_halves(float x) {
  const auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1]));
}
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int wave_min(int x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x = min(x, __shfl_xor(x, o));
  return uniform(x);
}
__device__ __forceinline__ int wave_max(int x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x = max(x, __shfl_xor(x, o));
  return uniform(x);
}

// First row of sequence s among all, cut to the call's rows.
__device__ __forceinline__ int first_row(const rkv_attend& a, int s) {
  return a.cu_q ? min(max(a.cu_q[s], 0), a.n_rows) : min(s, a.n_rows);
}

// Row tiles are numbered with room for a part-filled one per sequence: sequence s starts at floor(row0 G / 128) + s, which
// ascends and leaves each sequence ceil(rows / 128) numbers, so no list of tiles has to be built.
__device__ __forceinline__ int tile_start(const AttendLaunch& A, int row0, int s) { return row0 * A.group / kRows + s; }

// The first slot that position `at` (which may be negative) sees.
__device__ __forceinline__ int window_start(const rkv_attend& a, int at) { return a.window && at >= a.window ? at - a.window + 1 : 0; }

// The key tiles [t0, t1) that rows r0 .. r0 + 127 of a sequence of n_q tokens and n_kv slots may see (first_keys aside).
__device__ __forceinline__ void tile_span(const AttendLaunch& A, int seq, int r0, int n_q, int n_kv, int& t0, int& t1) {
  const rkv_attend& a = A.a;
  const int first = n_kv - n_q + div_by(r0, A.by_group), last = n_kv - n_q + min(n_q - 1, div_by(r0 + kRows - 1, A.by_group));
  int hi = n_kv;
  if (a.causal) hi = min(n_kv, max(last + 1, a.prefix_lens ? a.prefix_lens[seq] : 0));
  const int lo = window_start(a, first);
  t0 = lo / kKeys;
  t1 = max(t0, (hi + kKeys - 1) / kKeys);
}
__device__ __forceinline__ int slots_of(const AttendLaunch& A, int seq) {
  return min(max(A.a.lens[seq], 0), A.a.max_pages * A.p.page_size);
}
__device__ __forceinline__ int end_row(const rkv_attend& a, int seq) { return a.cu_q ? first_row(a, seq + 1) : min(seq + 1, a.n_rows); }

// A partial sum in the workspace: slot_rows rows of 128 floats (not divided by l), then pairs of what they and l are relative to
// (log2) and l; 16-byte aligned, slot_rows being even.
__device__ __forceinline__ float* part_slot(const AttendLaunch& A, int slot) {
  return A.parts + (size_t)slot * A.slot_rows * (kHeadDim + 2);
}

struct Bounds {   // of the waves
  int lo[4], all_lo[4], bad[4];
  int32_t ahead[4][64];   // page ids on their way
};
// The workgroup's LDS operations are done; vector memory operations stay in flight.
__device__ __forceinline__ void lds_sync() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt 0
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}
// Whether some wave of the workgroup says so.
__device__ __forceinline__ bool any_wave(Bounds& bounds, bool here) {
  const bool any = __any(here);
  if ((threadIdx.x & 63) == 0) bounds.bad[threadIdx.x >> 6] = any;
  lds_sync();
  const bool all = uniform(bounds.bad[0] | bounds.bad[1] | bounds.bad[2] | bounds.bad[3]);
  lds_sync();
  return all;
}
// Two 16-bit values.
template <bool kF16>
__device__ __forceinline__ f32x2 widen(uint32_t v) {
  if constexpr (kF16) return __builtin_convertvector(__builtin_bit_cast(f16x2, v), f32x2);
  else return f32x2{__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u)};
}

// Probability 0 times what a hidden slot holds is no 0 if that is infinite or NaN.  A tile whose rows see different slots and
// some of whose sums are not finite comes here (screening every tile of V instead cost packed documents 63 -> 80 us): if
// no slot that only some of its rows see is to blame, the sums stand; else its rows are summed up one by one, a wave
// each, two columns a lane, over the slots that they see and no others, and written: true.
template <bool kF16, bool kCap, bool kBias>
__device__ __forceinline__ bool attend_row_by_row(const AttendLaunch& A, Bounds& bounds, int seq, int row0, int n_q, int n_kv, int r0,
                                                  int h, int from, int to, int b_lo, int every_lo, int every_hi, int b_hi, float* part) {
  const rkv_attend& a = A.a;
  const rkv_pages& p = A.p;
  const int lane = threadIdx.x & 63, wv = uniform(threadIdx.x >> 6);
  const int32_t* table = a.table + seq * a.table_stride;
  const uint16_t* kp = static_cast<const uint16_t*>(p.k) + h * p.k_head + 2 * lane;
  const uint16_t* vp = static_cast<const uint16_t*>(p.v) + h * p.v_head + 2 * lane;
  auto place = [&](int key, int& page, int& at) {
    const int c = div_by(key, A.by_page);
    page = uniform(table[c]);
    at = key - c * p.page_size;
    return (uint32_t)page < (uint32_t)p.n_pages;
  };
  auto pair_at = [&](const uint16_t* x, int page, int at, int64_t page_stride, int64_t slot) {
    return widen<kF16>(*reinterpret_cast<const uint32_t*>(x + page * page_stride + at * slot));
  };
  bool blame = false;
  for (int part_of = 0; part_of < 2; ++part_of) {
    const int k0 = max(from, part_of ? max(b_lo, every_hi) : b_lo), k1 = min(to, part_of ? b_hi : min(b_hi, every_lo));
    for (int key = k0 + wv; key < k1; key += 4) {
      int page, at;
      if (!place(key, page, at)) continue;
      const f32x2 v = pair_at(vp, page, at, p.v_page, p.v_slot);
      blame |= v[0] * 0.f + v[1] * 0.f != 0.f;
    }
  }
  if (!any_wave(bounds, blame)) return false;
  const int n_rows = n_q * A.group, prefix = a.prefix_lens ? uniform(a.prefix_lens[seq]) : 0;
  const float cap2 = 2.f * kLog2e * a.softcap, in_cap = kCap ? 2.f * kLog2e * (a.scale / a.softcap) : 0.f;   // 1 / softcap may overflow
#pragma unroll 1
  for (int i = 0; i < 32; ++i) {
    const int mine = 32 * wv + i, r = r0 + mine;
    if (r >= n_rows) break;
    const int t = div_by(r, A.by_group), hq = h * A.group + r - t * A.group, pos = n_kv - n_q + t;
    const int64_t row = row0 + t;
    int hi = a.causal ? min(n_kv, max(pos + 1, prefix)) : n_kv, lo = window_start(a, pos);
    if (a.first_keys) lo = max(lo, uniform(a.first_keys[row]));
    lo = max(lo, from);
    hi = min(hi, to);
    const f32x2 q = widen<kF16>(*reinterpret_cast<const uint32_t*>(static_cast<const uint16_t*>(a.q) + row * a.q_token + hq * a.q_head + 2 * lane));
    const float slope = kBias ? a.slopes[hq] * kLog2e : 0.f;
    float m = -__builtin_inff(), l = 0.f, o0 = 0.f, o1 = 0.f;
#pragma unroll 1
    for (int key = lo; key < hi; ++key) {
      int page, at;
      f32x2 k = {0.f, 0.f}, v = {0.f, 0.f};
      if (place(key, page, at)) {
        k = pair_at(kp, page, at, p.k_page, p.k_slot);
        v = pair_at(vp, page, at, p.v_page, p.v_slot);
      }
      float x = fmaf(q[0], k[0], q[1] * k[1]);
#pragma unroll
      for (int s = 32; s > 0; s >>= 1) x += __shfl_xor(x, s);
      if constexpr (kCap) x = 0.5f * cap2 - cap2 / (1.f + __builtin_amdgcn_exp2f(in_cap * x));
      else x *= a.scale * kLog2e;
      if constexpr (kBias) x -= slope * fabsf((float)(pos - key));
      const float m2 = fmaxf(m, x), ref = m2 == -__builtin_inff() ? 0.f : m2;
      const float f = __builtin_amdgcn_exp2f(m - ref), e = __builtin_amdgcn_exp2f(x - ref);
      m = m2;
      l = fmaf(l, f, e);
      o0 = fmaf(o0, f, e * v[0]);
      o1 = fmaf(o1, f, e * v[1]);
    }
    if (part) {
      part[mine * kHeadDim + 2 * lane] = o0;
      part[mine * kHeadDim + 2 * lane + 1] = o1;
      part[A.slot_rows * kHeadDim + 2 * mine] = m;
      part[A.slot_rows * kHeadDim + 2 * mine + 1] = l;
    } else {
      const float inv = l == 0.f ? 0.f : 1.f / l;
      reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(a.out) + row * a.out_token + hq * a.out_head)[lane] = pack<kF16>(o0 * inv, o1 * inv);
      if (a.lse) a.lse[row * a.n_q_heads + hq] = row_lse(m, l);
    }
  }
  return true;
}

// kCap: capped scores, kBias: less a slope times the distance; kPage16: page_size % 16 = 0, pages less than 4 GiB and slots at least a
// row apart.  Key tiles t0 + u0 .. t0 + u0 + n - 1 of a row tile's span [t0, t1) (n < 0: all of them) for KV head h.  part: where the
// partial sums go, null: the rows are finished.
template <bool kF16, bool kCap, bool kBias, bool kPage16, bool kNarrow>
__device__ __forceinline__ void attend_rows(const AttendLaunch& A, unsigned char* smem, Bounds& bounds, int seq, int row0, int n_q,
                                            int n_kv, int r0, int h, int u0, int n, float* part) {
  const rkv_attend& a = A.a;
  const rkv_pages& p = A.p;
  int lane = threadIdx.x & 63;
  if constexpr (kNarrow) asm volatile("" : "+v"(lane));   // its addresses are not kept from one item to the next
  const int wv = uniform(threadIdx.x >> 6), col = lane & 31, half = lane >> 5;
  const int n_rows = n_q * A.group;

  // The slots a position sees, and a row's position.  Both bounds ascend with the row, so that those of the tile and of the
  // wave follow from their first and last rows, without a word from the other lanes: the first keys are requested at once.
  const int prefix = a.prefix_lens ? uniform(a.prefix_lens[seq]) : 0;
  auto hi_of = [&](int at) { return a.causal ? min(n_kv, max(at + 1, prefix)) : n_kv; };
  auto lo_of = [&](int at) { return window_start(a, at); };
  auto position = [&](int r) { return n_kv - n_q + div_by(min(r, n_rows - 1), A.by_group); };   // rows behind the last repeat it
  int b_lo = lo_of(position(r0)), b_hi = hi_of(position(r0 + kRows - 1));                       // slots some row sees
  const int w_first = kNarrow ? r0 : r0 + 32 * wv, w_last = kNarrow ? r0 + 15 : r0 + 32 * wv + 31;   // the wave's rows
  int all_lo = lo_of(position(w_last)), all_hi = hi_of(position(w_first));                      // every row of the wave
  int every_lo = lo_of(position(r0 + kRows - 1)), every_hi = hi_of(position(r0));               // every row of the tile
  const int r = min(w_first + (kNarrow ? lane & 15 : col), n_rows - 1);
  const int t = div_by(r, A.by_group), hq = h * A.group + r - t * A.group;
  const int64_t row = row0 + t;
  const int pos = n_kv - n_q + t;
  int lo = lo_of(pos), hi = hi_of(pos);
  if (a.first_keys) {   // these need not ascend
    lo = max(lo, a.first_keys[row]);
    all_lo = wave_max(lo);
    b_lo = wave_min(lo);
    every_lo = all_lo;
    if constexpr (!kNarrow) {
      if (lane == 0) {
        bounds.lo[wv] = b_lo;
        bounds.all_lo[wv] = all_lo;
      }
      __syncthreads();
      every_lo = uniform(max(max(bounds.all_lo[0], bounds.all_lo[1]), max(bounds.all_lo[2], bounds.all_lo[3])));
      b_lo = uniform(min(min(bounds.lo[0], bounds.lo[1]), min(bounds.lo[2], bounds.lo[3])));
    }
  }
  int t0, t1;
  tile_span(A, seq, r0, n_q, n_kv, t0, t1);
  if (n >= 0) {
    t0 += u0;
    t1 = min(t1, t0 + n);
  }
  t0 = max(t0, b_lo / kKeys);
  t1 = min(t1, (b_hi + kKeys - 1) / kKeys);

  // The four rows this lane fetches of a tile: 16 wv + 4 j + lane / 16, 16 bytes of each.  K rows lie in LDS with chunk c at
  // c ^ (row % 16), V rows with c at c ^ 4 (row % 4): the reads below then touch every bank alike.  Pages of a multiple of
  // 16 slots hold a wave's 16 rows in one: their addresses are a scalar base and offsets that never change (150 fewer vector
  // instructions a tile than with a page for each row, of 480).
  const uint32_t lds = lds_addr(smem);
  const int32_t* table = a.table + seq * a.table_stride;
  const auto* known = (const __attribute__((address_space(4))) int32_t*)(uintptr_t)table;   // scalar loads
  const char* kp = reinterpret_cast<const char*>(static_cast<const uint16_t*>(p.k) + h * p.k_head);
  const char* vp = reinterpret_cast<const char*>(static_cast<const uint16_t*>(p.v) + h * p.v_head);
  const int fr = lane >> 4;
  const uint32_t k_slot = (uint32_t)p.k_slot * 2, v_slot = (uint32_t)p.v_slot * 2;   // bytes; 15 of them stay below 2^32
  uint32_t k_off[4], v_off[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    k_off[j] = 16 * ((lane & 15) ^ (4 * j + fr));
    v_off[j] = 16 * ((lane & 15) ^ (4 * fr));
    if constexpr (kPage16) {   // not negative: slots are at least 256 bytes apart
      k_off[j] += (4 * j + fr) * k_slot - 1024 * j;
      v_off[j] += (4 * j + fr) * v_slot - 1024 * j;
    }
  }
  // Pages of a multiple of 16 slots: the page of the wave's rows of a tile (-1: not visible) and the slot in it.
  struct Place {
    int page, at;
  };
  // Others: lane i looks up row i % 16 of tile i / 16 of four, the next four ahead, and the addresses go round by permutes
  // (looking up every row of a tile by itself took 512 tokens after 32K from 286 to 340 us).
  int page4 = -1;
  const char *k4 = nullptr, *v4 = nullptr;
  const uint32_t ahead = lds_addr(bounds.ahead[wv]);
  auto key4 = [&](int tl) { return (tl + fr) * kKeys + 16 * wv + (lane & 15); };
  auto look = [&](int tl) __attribute__((always_inline)) {
    dma4(table + div_by(min(max(key4(tl), b_lo), b_hi - 1), A.by_page), ahead);   // no register waits for it
  };
  const char* zeros = reinterpret_cast<const char*>(zero_row);
  auto row4 = [&](int tl, const char* rows, int64_t page_stride, uint32_t slot) __attribute__((always_inline)) {
    const int key = key4(tl);
    const bool in = key >= b_lo && key < b_hi && (uint32_t)page4 < (uint32_t)p.n_pages;
    const int at = key - div_by(in ? key : 0, A.by_page) * p.page_size;
    return in ? rows + (uint64_t)(uint32_t)page4 * (uint64_t)(2 * page_stride) + (uint64_t)(uint32_t)at * slot : zeros;
  };
  auto find = [&](int tl, Place& x) __attribute__((always_inline)) {
    if constexpr (kPage16) {
      const int key = tl * kKeys + 16 * wv;
      const bool in = key + 16 > b_lo && key < b_hi;
      const int c = div_by(in ? key : 0, A.by_page);
      x.at = key - c * p.page_size;
      x.page = in ? known[c] : -1;
    }
  };
  auto fetch = [&](int tl, const Place& x, const char* rows, const char* rows4, int64_t page_stride, uint32_t slot, const uint32_t (&off)[4],
                   uint32_t to) __attribute__((always_inline)) {
    to += lds + wv * 4096;
    if constexpr (kPage16) {
      const int key = tl * kKeys + 16 * wv;
      const uint32_t pg = x.page;
      const bool held = pg < (uint32_t)p.n_pages;
      const char* src = rows + (uint64_t)pg * (uint32_t)(2 * page_stride) + (uint64_t)(uint32_t)x.at * slot;
      if (held && key >= b_lo && key + 16 <= b_hi) {
        dma16s_four(src, off, to);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const bool in = held && key + 4 * j + fr >= b_lo && key + 4 * j + fr < b_hi;
          dma16(in ? src + (off[j] + 1024 * j) : zeros + (off[j] & 240), to + 1024 * j);
        }
      }
    } else {
      const int from = 4 * (16 * ((tl - t0) & 3) + fr);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t x0 = __builtin_amdgcn_ds_bpermute(from + 16 * j, (int)(uint32_t)(uintptr_t)rows4);
        const uint32_t x1 = __builtin_amdgcn_ds_bpermute(from + 16 * j, (int)(uint32_t)((uintptr_t)rows4 >> 32));
        dma16(reinterpret_cast<const char*>((uintptr_t)x1 << 32 | x0) + off[j], to + 1024 * j);
      }
    }
  };
  // Of each four tiles from t0, K's first is requested before V's, and V's before K's fifth.
  auto fetch_k = [&](int tl, const Place& x, int buf) __attribute__((always_inline)) {
    if constexpr (!kPage16) {
      if (((tl - t0) & 3) == 0) {
        page4 = bounds.ahead[wv][lane];   // requested four tiles ago
        asm volatile("" : "+v"(page4));
        __builtin_amdgcn_s_waitcnt(0xc07f);   // read before the next ones may arrive
        k4 = row4(tl, kp, p.k_page, k_slot);
        if (tl + 4 < t1) look(tl + 4);
      }
    }
    fetch(tl, x, kp, k4, p.k_page, k_slot, k_off, buf * kTileBytes);
  };
  auto fetch_v = [&](int tl, const Place& x, int buf) __attribute__((always_inline)) {
    if constexpr (!kPage16) {
      if (((tl - t0) & 3) == 0) v4 = row4(tl, vp, p.v_page, v_slot);
    }
    fetch(tl, x, vp, v4, p.v_page, v_slot, v_off, (2 + buf) * kTileBytes);
  };
  if constexpr (!kPage16) {
    if (t0 < t1) {
      look(t0);
      wait_vmcnt<0>();
      asm volatile("" ::: "memory");
    }
  }

  const float sl2 = fmaxf(fabsf(a.scale) * kLog2e, 1e-30f);   // a negative scale's sign is in q; above 0, so that hidden stays hidden
  const float slope = kBias ? a.slopes[hq] * kLog2e : 0.f;
  const float cap2 = 2.f * kLog2e * a.softcap, in_cap = kCap ? 2.f * sl2 / a.softcap : 0.f;
  // A product becomes what is compared and exponentiated: the score is grow x + base, in log2 units, with grow >= 0.
  //   neither: x = the product, the scale in grow;
  //   capped:  c tanh(y / c) = c - 2 c / (1 + exp(2 y / c)): x = -1 / (1 + exp(2 y / c)), grow = 2 c, base = c;
  //   biased (after the cap): x = the score.  far: the distance of the row from the lane's first key, key: from there.
  auto score = [&](float y, int key, float far) __attribute__((always_inline)) {
    if constexpr (kCap) y = __builtin_amdgcn_rcpf(-1.f - __builtin_amdgcn_exp2f(y * in_cap));
    if constexpr (kBias) {
      y = kCap ? fmaf(y, cap2, 0.5f * cap2) : y * sl2;
      y = fmaf(-slope, fabsf(far - (float)key), y);
    }
    return y;
  };
  const float grow = kBias ? 1.f : kCap ? cap2 : sl2, base = !kBias && kCap ? 0.5f * cap2 : 0.f;
  const uint16_t* qrow = static_cast<const uint16_t*>(a.q) + row * a.q_token + hq * a.q_head;
  float m = -__builtin_inff(), l = 0.f, ref = 0.f;   // ref: the running maximum less kUnder, 0 while there is none

  if constexpr (kNarrow) {
    // At most 16 rows, all of them in every wave; a wave takes the 16 keys of each tile that it fetched itself, two tiles
    // ahead, and waits for no other: 16x16x32 and 16x16x16 MFMA, a lane holds keys 4 (lane / 16) + 0..3 of row lane % 16.
    const int l16 = lane & 15, lg = lane >> 4;
    Place next;
    auto fetch_both = [&](int tl, int buf) __attribute__((always_inline)) {
      fetch_k(tl, next, buf);
      fetch_v(tl, next, buf);
    };
    if (t0 < t1) {
      find(t0, next);
      fetch_both(t0, 0);
      if (t0 + 1 < t1) {
        find(t0 + 1, next);
        fetch_both(t0 + 1, 1);
      }
      if (t0 + 2 < t1) find(t0 + 2, next);
    }
    u32x4 q[4];
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      q[s] = *reinterpret_cast<const u32x4*>(qrow + 32 * s + 8 * lg);
      if (a.scale < 0.f) q[s] ^= 0x80008000u;
    }
    const uint32_t k_at = lds + wv * 4096 + l16 * 256;
    const uint32_t v_at = lds + 2 * kTileBytes + wv * 4096 + (4 * lg + (l16 >> 2)) * 256 + (l16 & 1) * 8;
    f32x4 o[8] = {};
#pragma unroll 1
    for (int tl = t0; tl < t1; ++tl) {
      const uint32_t buf = ((tl - t0) & 1) * kTileBytes;
      if (tl + 1 < t1) wait_vmcnt<8>();   // the next tile may be in flight
      else wait_vmcnt<0>();
      asm volatile("" ::: "memory");
      u32x4 kf[4];
      u32x2 vf[8];
#pragma unroll
      for (int s = 0; s < 4; ++s) kf[s] = lds_read16(k_at + buf + ((4 * s + lg) ^ l16) * 16);
#pragma unroll
      for (int d = 0; d < 8; ++d) vf[d] = lds_read_tr(v_at + buf + ((2 * d + ((l16 & 3) >> 1)) ^ (4 * (l16 >> 2))) * 16);
      // The whole tile is in registers before the first product, and its memory free for the tile after the next, whose
      // fetch then runs under the softmax: one token after 4096 in one workgroup a head 41 -> 35 us.
      asm volatile("" ::: "memory");
      __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt 0
      f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < 4; ++s) x = mma16<kF16>(kf[s], q[s], x);
      if (tl + 2 < t1) {
        fetch_both(tl + 2, (tl - t0) & 1);
        if (tl + 3 < t1) find(tl + 3, next);
      }
      const int key0 = tl * kKeys + 16 * wv;
      const float far = (float)(pos - key0 - 4 * lg);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = score(x[i], i, far);
      if (key0 < all_lo || key0 + 16 > all_hi) {
        const int from = lo - key0 - 4 * lg, to = hi - key0 - 4 * lg;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (i < from || i >= to) x[i] = -__builtin_inff();
      }
      float top = fmaf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), grow, base);
      if (__any(top > m + kGrow)) {   // the row's, over its four lanes
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float m2 = fmaxf(m, top), f = m2 > m ? __builtin_amdgcn_exp2f(m - m2) : 1.f;
        m = m2;
        ref = m == -__builtin_inff() ? 0.f : m - kUnder<kF16>;
        l *= f;
#pragma unroll
        for (int d = 0; d < 8; ++d)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[d][i] *= f;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[i] = __builtin_amdgcn_exp2f(fmaf(x[i], grow, base - ref));
        l += x[i];
      }
      const u32x2 pr = {pack<kF16>(x[0], x[1]), pack<kF16>(x[2], x[3])};
#pragma unroll
      for (int d = 0; d < 8; ++d)
        o[d] = mma16s<kF16>(vf[d], pr, o[d]);
    }
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    // The four waves' sums meet by way of the memory each fetched into: columns below 64 in its part of K's first tile, the
    // others in the second's, chunks of 16 bytes at c ^ row; m and l in V's first.
#pragma unroll
    for (int d = 0; d < 8; ++d)
      *(__attribute__((address_space(3))) f32x4*)(uintptr_t)(k_at + (d >> 2) * kTileBytes + ((4 * (d & 3) + lg) ^ l16) * 16) = o[d];
    if (lg == 0) *(__attribute__((address_space(3))) f32x2*)(uintptr_t)(lds + 2 * kTileBytes + wv * 4096 + l16 * 8) = f32x2{m, l};
    lds_sync();
    const int x = 4 * wv + lg, c = l16;      // this thread's row and eight columns
    f32x2 ml[4];
    float mm = -__builtin_inff(), ll = 0.f, sum[8] = {};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      ml[w] = *(const __attribute__((address_space(3))) f32x2*)(uintptr_t)(lds + 2 * kTileBytes + w * 4096 + x * 8);
      mm = fmaxf(mm, ml[w][0]);
    }
    const float mr = mm == -__builtin_inff() ? 0.f : mm;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float f = __builtin_amdgcn_exp2f(ml[w][0] - mr);
      ll = fmaf(ml[w][1], f, ll);
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const f32x4 v = *(const __attribute__((address_space(3))) f32x4*)(uintptr_t)(lds + (c >> 3) * kTileBytes + w * 4096 + x * 256 +
                                                                                     ((2 * (c & 7) + u) ^ x) * 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[4 * u + i] = fmaf(v[i], f, sum[4 * u + i]);
      }
    }
    mm -= kUnder<kF16>;   // what the sums are relative to
    if (b_lo != every_lo || b_hi != every_hi) {
      float finite = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) finite = fmaf(sum[i], 0.f, finite);
      if (any_wave(bounds, finite != 0.f) &&   // NaN
          attend_row_by_row<kF16, kCap, kBias>(A, bounds, seq, row0, n_q, n_kv, r0, h, t0 * kKeys, t1 * kKeys, b_lo, every_lo, every_hi, b_hi, part))
        return;
    }
    if (r0 + x >= n_rows) return;
    if (part) {
#pragma unroll
      for (int u = 0; u < 2; ++u)
        *reinterpret_cast<f32x4*>(part + x * kHeadDim + 8 * c + 4 * u) = f32x4{sum[4 * u], sum[4 * u + 1], sum[4 * u + 2], sum[4 * u + 3]};
      if (c == 0) *reinterpret_cast<f32x2*>(part + A.slot_rows * kHeadDim + 2 * x) = f32x2{mm, ll};
      return;
    }
    const float inv = ll == 0.f ? 0.f : 1.f / ll;
    const int token = div_by(r0 + x, A.by_group), head = h * A.group + r0 + x - token * A.group;
    *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(a.out) + (row0 + token) * a.out_token + head * a.out_head + 8 * c) =
        u32x4{pack<kF16>(sum[0] * inv, sum[1] * inv), pack<kF16>(sum[2] * inv, sum[3] * inv), pack<kF16>(sum[4] * inv, sum[5] * inv),
              pack<kF16>(sum[6] * inv, sum[7] * inv)};
    if (a.lse && c == 0) a.lse[(int64_t)(row0 + token) * a.n_q_heads + head] = row_lse(mm, ll);
  } else {

  // Iteration tl needs tile tl of V and tile tl + 1 of K, requested in the iteration before; K's tiles are in buffers
  // (tl - t0) % 2, V's in 2 + (tl - t0) % 2.
  Place here, next;
  auto advance = [&](int tl, int b) __attribute__((always_inline)) {   // b = (tl + 1 - t0) % 2
    tile_sync();
    if (tl + 2 < t1) fetch_k(tl + 2, next, 1 - b);
    if (tl + 1 < t1 && tl >= t0) fetch_v(tl + 1, here, b);
    here = next;
    if (tl + 3 < t1) find(tl + 3, next);
  };
  if (t0 < t1) {
    find(t0, here);
    if (t0 + 1 < t1) find(t0 + 1, next);
    fetch_k(t0, here, 0);
    fetch_v(t0, here, 0);
  }
  u32x4 q[8];
#pragma unroll
  for (int s = 0; s < 8; ++s) q[s] = *reinterpret_cast<const u32x4*>(qrow + 16 * s + 8 * half);
  if (a.scale < 0.f) {
#pragma unroll
    for (int s = 0; s < 8; ++s) q[s] ^= 0x80008000u;
  }

  f32x16 o[4] = {};
  uint32_t k_lane[8], v_lane[4];
#pragma unroll
  for (int st = 0; st < 8; ++st) k_lane[st] = lds + col * 256 + (((2 * st) ^ (col & 15) ^ half) * 16);
  // V^T: lane reads 4 columns of key 4 half + (lane % 16) / 4 (+ 8), chunk 4 d + 2 ((lane / 16) % 2) + (lane % 4) / 2
  const int v_key = 4 * half + ((lane & 15) >> 2);
#pragma unroll
  for (int d = 0; d < 4; ++d)
    v_lane[d] = lds + v_key * 256 + ((4 * d + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ (4 * (v_key & 3))) * 16 + (lane & 1) * 8;

  f32x16 sa[2], sb[2];  // scores of a tile and the next: s.[u][i] is key 32 u + 8 (i / 4) + 4 half + i % 4
  u32x4 pr[4];          // probabilities of a tile, 16 keys each

  auto k_frag = [&](int i, uint32_t kb) __attribute__((always_inline)) { return lds_read16(k_lane[i & 7] + kb + (i >> 3) * 8192); };
  auto key_of = [](int i) { return 32 * (i >> 4) + 8 * ((i & 15) >> 2) + (i & 3); };   // of score i of 32, from 4 half
  auto distance = [&](int tl) __attribute__((always_inline)) { return (float)(pos - tl * kKeys - 4 * half); };   // of key 4 half
  // A tile that a row sees part of: the scores of the others, and the maximum again.
  auto hide = [&](int tl, f32x16 (&x)[2], float& top) __attribute__((always_inline)) {
    const int key0 = tl * kKeys;
    if (key0 >= all_lo && key0 + kKeys <= all_hi) return;
    const int from = lo - key0 - 4 * half, to = hi - key0 - 4 * half;
    top = -__builtin_inff();
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int key = 32 * u + 8 * (i >> 2) + (i & 3);
        if (key < from || key >= to) x[u][i] = -__builtin_inff();
        top = fmaxf(top, x[u][i]);
      }
  };
  // The maximum of a tile's scores joins the running one; what has been summed is rescaled if it grew by much.
  auto settle = [&](float top) __attribute__((always_inline)) {
    top = fmaf(max_halves(top), grow, base);
    if (__any(top > m + kGrow)) {
      const float m2 = fmaxf(m, top), f = m2 > m ? __builtin_amdgcn_exp2f(m - m2) : 1.f;
      m = m2;
      ref = m == -__builtin_inff() ? 0.f : m - kUnder<kF16>;
      l *= f;
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] *= f;
    }
  };
  // Scores of the first tile.
  auto begin = [&](int tl, f32x16 (&x)[2], uint32_t kb) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i >> 3] = mma32<kF16>(k_frag(i, kb), q[i & 7], (i & 7) == 0 ? f32x16{} : x[i >> 3]);
    const float far = distance(tl);
    float top = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      x[i >> 4][i & 15] = score(x[i >> 4][i & 15], key_of(i), far);
      top = fmaxf(top, x[i >> 4][i & 15]);
    }
    hide(tl, x, top);
    settle(top);
  };
  // Probabilities 2 i and 2 i + 1 of a tile.
  auto pair = [&](const f32x16 (&x)[2], int i) __attribute__((always_inline)) {
    float e[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const float z = x[i >> 3][2 * (i & 7) + j];
      e[j] = __builtin_amdgcn_exp2f(fmaf(z, grow, base - ref));
      l += e[j];
    }
    pr[i >> 2][i & 3] = pack<kF16>(e[0], e[1]);
  };
  // Tile tl, whose scores are x, summed up, and the next one's scores y: the probabilities are computed between the products
  // of K and V, the next maximum between those of V, so that both pipes have work of this wave at any time.  The last tile's
  // "next" is whatever lies in LDS, and goes nowhere.
  auto sum_up = [&](int tl, f32x16 (&x)[2], f32x16 (&y)[2], uint32_t kb, uint32_t vb) __attribute__((always_inline)) {
    {
      u32x4 f[4];
#pragma unroll
      for (int i = 0; i < 3; ++i) f[i] = k_frag(i, kb);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        if (i + 3 < 16) f[(i + 3) & 3] = k_frag(i + 3, kb);
        y[i >> 3] = mma32<kF16>(f[i & 3], q[i & 7], (i & 7) == 0 ? f32x16{} : y[i >> 3]);
        if (i * kAhead / 16 != (i + 1) * kAhead / 16) pair(x, i * kAhead / 16);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    const float far = distance(tl + 1);
    float top = -__builtin_inff();
    {
      auto v_frag = [&](int i) __attribute__((always_inline)) {   // 16 keys i / 4, columns 32 (i % 4) ..
        const u32x2 v0 = lds_read_tr(v_lane[i & 3] + vb + (i >> 2) * 4096);
        const u32x2 v1 = lds_read_tr(v_lane[i & 3] + vb + (i >> 2) * 4096 + 2048);
        return u32x4{v0[0], v0[1], v1[0], v1[1]};
      };
      u32x4 f[4];
#pragma unroll
      for (int i = 0; i < 3; ++i) f[i] = v_frag(i);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        if (i + 3 < 16) f[(i + 3) & 3] = v_frag(i + 3);
        o[i & 3] = mma32<kF16>(f[i & 3], pr[i >> 2], o[i & 3]);
        if (kAhead + i < 16) pair(x, kAhead + i);
        y[i >> 3][2 * (i & 7)] = score(y[i >> 3][2 * (i & 7)], key_of(2 * i), far);
        y[i >> 3][2 * (i & 7) + 1] = score(y[i >> 3][2 * (i & 7) + 1], key_of(2 * i + 1), far);
        top = fmaxf(fmaxf(top, y[i >> 3][2 * (i & 7)]), y[i >> 3][2 * (i & 7) + 1]);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    if (tl + 1 < t1) {
      hide(tl + 1, y, top);
      settle(top);
    }
  };
  if (t0 < t1) {
    if (r0 + 32 * wv < n_rows) {
      advance(t0 - 1, 0);
      begin(t0, sa, 0);
#pragma unroll 1
      for (int tl = t0;; tl += 2) {
        advance(tl, 1);
        sum_up(tl, sa, sb, kTileBytes, 2 * kTileBytes);
        if (tl + 1 >= t1) break;
        advance(tl + 1, 0);
        sum_up(tl + 1, sb, sa, 0, 3 * kTileBytes);
        if (tl + 2 >= t1) break;
      }
    } else {      // no rows: this wave fetches for the others
#pragma unroll 1
      for (int tl = t0 - 1; tl < t1; ++tl) advance(tl, (tl + 1 - t0) & 1);
    }
  }
  __syncthreads();   // bounds and tiles are free for the next rows
  if (b_lo != every_lo || b_hi != every_hi) {
    float finite = 0.f;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) finite = fmaf(o[d][i], 0.f, finite);
    if (any_wave(bounds, finite != 0.f) &&   // NaN
        attend_row_by_row<kF16, kCap, kBias>(A, bounds, seq, row0, n_q, n_kv, r0, h, t0 * kKeys, t1 * kKeys, b_lo, every_lo, every_hi, b_hi, part))
      return;
  }

  l += __shfl_xor(l, 32);
  m -= kUnder<kF16>;   // what the sums are relative to
  // The wave's rows by way of its quarter of the tiles' memory, chunks of 16 bytes at c ^ row: whole rows leave it.
  const int rows = min(32, n_rows - r0 - 32 * wv);
  if (rows <= 0) return;
  uint32_t ln = lane;
  asm volatile("" : "+v"(ln));   // addresses of this end are not kept from one item to the next
  const uint32_t mem = lds + wv * 16384, cl = ln & 31, hf = ln >> 5;
  if (part) {
    const uint32_t to = mem + cl * 512;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *(__attribute__((address_space(3))) f32x4*)(uintptr_t)(to + ((8 * d + 2 * i + hf) ^ cl) * 16) =
            f32x4{o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]};
#pragma unroll 2
    for (uint32_t x = hf; x < (uint32_t)rows; x += 2)
      *reinterpret_cast<u32x4*>(part + (32 * wv + x) * kHeadDim + 4 * cl) = lds_read16(mem + x * 512 + (cl ^ x) * 16);
    if (hf == 0 && cl < (uint32_t)rows) *reinterpret_cast<f32x2*>(part + A.slot_rows * kHeadDim + 2 * (32 * wv + cl)) = f32x2{m, l};
    return;
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  const uint32_t to = mem + cl * 256 + hf * 8;
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *(__attribute__((address_space(3))) u32x2*)(uintptr_t)(to + ((4 * d + i) ^ (cl & 15)) * 16) =
          u32x2{pack<kF16>(o[d][4 * i] * inv, o[d][4 * i + 1] * inv), pack<kF16>(o[d][4 * i + 2] * inv, o[d][4 * i + 3] * inv)};
#pragma unroll 2
  for (uint32_t x = ln >> 4; x < (uint32_t)rows; x += 4) {
    const int at = r0 + 32 * wv + (int)x, token = div_by(at, A.by_group), head = h * A.group + at - token * A.group;
    *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(a.out) + (row0 + token) * a.out_token + head * a.out_head + 8 * (ln & 15)) =
        lds_read16(mem + x * 256 + ((ln & 15) ^ (x & 15)) * 16);
  }
  if (a.lse && hf == 0 && cl < (uint32_t)rows) {
    const int at = r0 + 32 * wv + (int)cl, token = div_by(at, A.by_group), head = h * A.group + at - token * A.group;
    a.lse[(int64_t)(row0 + token) * a.n_q_heads + head] = row_lse(m, l);
  }
  }   // !kNarrow
}

// At most 16 rows go the narrow way.
template <bool kF16, bool kCap, bool kBias, bool kPage16>
__device__ __forceinline__ void attend_tile(const AttendLaunch& A, unsigned char* smem, Bounds& bounds, int seq, int row0, int n_q,
                                            int n_kv, int r0, int h, int u0, int n, float* part) {
  if (n_q * A.group - r0 <= 16) attend_rows<kF16, kCap, kBias, kPage16, true>(A, smem, bounds, seq, row0, n_q, n_kv, r0, h, u0, n, part);
  else attend_rows<kF16, kCap, kBias, kPage16, false>(A, smem, bounds, seq, row0, n_q, n_kv, r0, h, u0, n, part);
}

// The same for sequences of more than one tile alone, when those are few: floor(rows / 128) >= 1 then, and twice that is room
// enough, so that s can start at 2 floor(row0 G / 128).
__device__ __forceinline__ int long_start(const AttendLaunch& A, int row0, int s) {
  return A.few_long ? 2 * (row0 * A.group / kRows) : tile_start(A, row0, s);
}
// The sequence of a tile numbered by long_start: 64-way bisection by a wave.
__device__ __forceinline__ int tile_sequence(const AttendLaunch& A, int tile) {
  int lo = 0, n = A.a.n_seqs;
  while (n > 1) {
    const int step = (n + 63) / 64, at = (int)(threadIdx.x & 63) * step;
    const uint64_t in = __ballot(at < n && long_start(A, first_row(A.a, lo + at), lo + at) <= tile);
    const int k = max(0, (int)__popcll(in) - 1) * step;
    lo += k;
    n = min(step, n - k);
  }
  return lo;
}

// One workgroup per row tile and KV head.  First the sequences of one tile (decoding ones, whose keys may be many), then the
// others' tiles, the longest of a causal prompt first.  (With the decoding sequences in their own places, 24 of them before
// four prompts were the last to begin: 325 us against 301.  With all sequences' last tiles first, the tiles of a head that
// read the same keys come apart: 512 tokens of eight sequences after 3584 took 293 us against 262.)
template <bool kF16, bool kCap, bool kBias, bool kPage16>
__global__ __launch_bounds__(256, 2) void attend_tiles_kernel(const AttendLaunch A) {
  __shared__ __align__(1024) unsigned char smem[4 * kTileBytes];   // [buffer][K, V]
  __shared__ Bounds bounds;
  const int place = blockIdx.x / A.p.n_kv_heads, h = blockIdx.x - place * A.p.n_kv_heads;
  const bool brief = place < A.a.n_seqs;
  const int tile = A.n_places - 1 - place, seq = brief ? place : uniform(tile_sequence(A, tile));
  const int row0 = uniform(first_row(A.a, seq)), n_q = uniform(end_row(A.a, seq)) - row0, n_rows = n_q * A.group;
  const int r0 = brief ? 0 : (tile - long_start(A, row0, seq)) * kRows;
  if ((n_rows <= kRows) != brief || r0 < 0 || r0 >= n_rows) return;
  attend_tile<kF16, kCap, kBias, kPage16>(A, smem, bounds, seq, row0, n_q, uniform(slots_of(A, seq)), r0, h, 0, -1, nullptr);
}

// The list of row tiles that every workgroup of attend_shares_kernel makes.
struct List {
  int32_t row0[kListed + 1];     // first row of each sequence
  int32_t slots[kListed];        // of each sequence
  int32_t before[kListed + 1];   // key tiles of a head before row tile i
  uint16_t seq[kListed];         // sequence of row tile i
  int32_t wave[4];
};
constexpr int kPer = kListed / 256;   // row tiles of a thread

// Fills the list; the key tiles of a head, fewer than 2^31 (the host lets no other call here).
__device__ __forceinline__ int make_list(const AttendLaunch& A, List& L) {
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, n = A.a.n_seqs;
  for (int s = tid; s <= n; s += 256) L.row0[s] = s < n ? first_row(A.a, s) : end_row(A.a, n - 1);
  for (int s = tid; s < n; s += 256) L.slots[s] = slots_of(A, s);
  __syncthreads();
  int cost[kPer];
  int sum = 0;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int tile = tid * kPer + i;
    cost[i] = 0;
    if (tile < A.n_tiles) {
      int lo = 0, hi = n;
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (tile_start(A, L.row0[mid], mid) <= tile) lo = mid;
        else hi = mid;
      }
      L.seq[tile] = (uint16_t)lo;
      const int n_q = L.row0[lo + 1] - L.row0[lo], r0 = (tile - tile_start(A, L.row0[lo], lo)) * kRows;
      if (r0 >= 0 && r0 < n_q * A.group) {
        int t0, t1;
        tile_span(A, lo, r0, n_q, L.slots[lo], t0, t1);
        cost[i] = max(1, t1 - t0);   // rows that see nothing are written too
      }
    }
    sum += cost[i];
  }
  int x = sum;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(x, o);
    if (lane >= o) x += y;
  }
  if (lane == 63) L.wave[wv] = x;
  __syncthreads();
  int before = x - sum;
  for (int i = 0; i < wv; ++i) before += L.wave[i];
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    L.before[tid * kPer + i] = before;
    before += cost[i];
  }
  if (tid == 255) L.before[kListed] = before;
  const int all = uniform(L.wave[0] + L.wave[1] + L.wave[2] + L.wave[3]);
  __syncthreads();
  return all;
}

// kShares workgroups with an equal share each of all items' key tiles, in the order (head, row tile, key tile).  Workgroup b
// runs on XCD b % 8: it takes share (b % 8) kShares / 8 + b / 8, so that the row tiles of a head, which read the same
// keys, meet in one L2.
template <bool kF16, bool kCap, bool kBias, bool kPage16>
__global__ __launch_bounds__(256, 2) void attend_shares_kernel(const AttendLaunch A) {
  __shared__ __align__(1024) unsigned char smem[4 * kTileBytes];
  __shared__ Bounds bounds;
  __shared__ List L;
  const int tid = threadIdx.x;
  const int all = make_list(A, L);
  const int w = (int)(blockIdx.x % 8) * (kShares / 8) + (int)blockIdx.x / 8;
  i32x4 record = {0, 0, 0, 0};   // parts + 1024 head, sequence's first row, first row of the tile, rows of the sequence
  const int64_t total = (int64_t)all * A.p.n_kv_heads;
  const int64_t share = max((int64_t)A.least, (total + kShares - 1) / kShares);
  int64_t pos = w * share;
  const int64_t end = min(total, pos + share);
  while (pos < end) {
    const int h = uniform((int)(pos / all)), rem = uniform((int)(pos - (int64_t)h * all));
    int lo = 0, hi = kListed;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (L.before[mid] <= rem) lo = mid;
      else hi = mid;
    }
    const int tile = uniform(lo), seq = uniform(L.seq[tile]);
    const int u0 = rem - uniform(L.before[tile]), count = uniform(L.before[tile + 1]) - uniform(L.before[tile]);
    const int n = (int)min((int64_t)(count - u0), end - pos);
    const int row0 = uniform(L.row0[seq]), n_q = uniform(L.row0[seq + 1]) - row0, r0 = (tile - tile_start(A, row0, seq)) * kRows;
    float* part = nullptr;
    if (n < count) {
      part = part_slot(A, 2 * w + (u0 == 0));
      if (u0 == 0) {
        record = i32x4{(int)((pos + count - 1) / share) - w + 1 + 1024 * h, row0, r0, n_q * A.group};
      }
    }
    attend_tile<kF16, kCap, kBias, kPage16>(A, smem, bounds, seq, row0, n_q, uniform(L.slots[seq]), r0, h, u0, n, part);
    lds_sync();   // the memory that rows left by is the next tiles'
    pos += n;
  }
  if (tid == 0) reinterpret_cast<i32x4*>(A.records)[w] = record;
}

// The parts of the items that begin in one share and end in a later one.  Which these are is in the records; the workgroups
// share out their rows, 8 at a time or fewer where items are few.  32 lanes hold the 128 values of a row; with fewer than 8
// rows, several such groups take a row's parts in turn and meet in LDS.
constexpr int kJoinThreads = 256, kJoinGrid = 1024;
template <bool kF16>
__global__ __launch_bounds__(kJoinThreads) void join_kernel(const AttendLaunch A) {
  __shared__ f32x4 sO[8][32];
  __shared__ float sM[8], sL[8];
  __shared__ i32x4 sRecord[kShares];
  __shared__ int sItem[kShares], sCount[4], sRows[4];
  static_assert(kShares == 2 * kJoinThreads, "two records a thread");
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  const i32x4 first = reinterpret_cast<const i32x4*>(A.records)[2 * tid], second = reinterpret_cast<const i32x4*>(A.records)[2 * tid + 1];
  const bool one = first[0] != 0, two = second[0] != 0;
  const int widest = wave_max(max(one ? min(kRows, first[3] - first[2]) : 0, two ? min(kRows, second[3] - second[2]) : 0));
  const uint64_t ones = __ballot(one), twos = __ballot(two), below = (uint64_t(1) << lane) - 1;
  if (lane == 0) {
    sCount[wv] = (int)(__popcll(ones) + __popcll(twos));
    sRows[wv] = widest;
  }
  __syncthreads();
  int at = 0, items = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (i == wv) at = items;
    items += sCount[i];
  }
  at += (int)(__popcll(ones & below) + __popcll(twos & below));
  if (one) {
    sRecord[at] = first;
    sItem[at++] = 2 * tid;
  }
  if (two) {
    sRecord[at] = second;
    sItem[at] = 2 * tid + 1;
  }
  items = uniform(items);
  const int rows_most = uniform(max(max(sRows[0], sRows[1]), max(sRows[2], sRows[3])));
  int most = 8, chunks = (rows_most + 7) / 8;   // rows of a workgroup at once
  while (most > 1 && items * chunks < kJoinGrid) {
    most >>= 1;
    chunks = (rows_most + most - 1) / most;
  }
  const rkv_attend& a = A.a;
  const int grp = tid >> 5, c = tid & 31;
  for (int task = blockIdx.x; task < items * chunks; task += kJoinGrid) {
    __syncthreads();   // the list is whole; sO is free
    const int w = uniform(sItem[task / chunks]), y0 = task % chunks * most;
    const i32x4 record = sRecord[task / chunks];
    const int parts = uniform(record[0] & 1023), h = uniform(record[0] >> 10), row0 = uniform(record[1]), r0 = uniform(record[2]);
    const int rows = min(most, min(kRows, uniform(record[3]) - r0) - y0);
    if (rows <= 0) continue;
    const int each = 8 / rows;                        // groups of a row
    const int i = grp / each, g = grp - i * each;     // row, and place among its groups
    const bool in = i < rows;
    const int k = y0 + (in ? i : 0);
    float m = -__builtin_inff(), l = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    auto add = [&](float m2, float l2, f32x4 v) {
      const float top = fmaxf(m, m2), ref = top == -__builtin_inff() ? 0.f : top;
      const float f = __builtin_amdgcn_exp2f(m - ref), f2 = __builtin_amdgcn_exp2f(m2 - ref);
      m = top;
      l = l * f + l2 * f2;
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] = acc[e] * f + v[e] * f2;
    };
    for (int j0 = g; j0 < parts; j0 += 4 * each) {   // four parts in flight
      f32x2 ml[4];
      f32x4 v[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int jj = min(j0 + j * each, parts - 1);
        const float* from = part_slot(A, jj ? 2 * (w + jj) : 2 * w + 1);
        ml[j] = *reinterpret_cast<const f32x2*>(from + A.slot_rows * kHeadDim + 2 * k);   // m, l
        v[j] = *reinterpret_cast<const f32x4*>(from + k * kHeadDim + 4 * c);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (j0 + j * each < parts) add(ml[j][0], ml[j][1], v[j]);
    }
    sO[grp][c] = acc;
    if (c == 0) {
      sM[grp] = m;
      sL[grp] = l;
    }
    __syncthreads();
    if (!in || g) continue;
    for (int x = 1; x < each; ++x) add(sM[grp + x], sL[grp + x], sO[grp + x][c]);
    const int r = r0 + k, t = div_by(r, A.by_group), hq = h * A.group + r - t * A.group;
    const int64_t row = row0 + t;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    uint16_t* out = static_cast<uint16_t*>(a.out) + row * a.out_token + hq * a.out_head + 4 * c;
    *reinterpret_cast<u32x2*>(out) = u32x2{pack<kF16>(acc[0] * inv, acc[1] * inv), pack<kF16>(acc[2] * inv, acc[3] * inv)};
    if (a.lse && c == 0) a.lse[row * a.n_q_heads + hq] = row_lse(m, l);
  }
}

template <bool kF16, bool kCap, bool kBias, bool kPage16>
void launch_kernels(const AttendLaunch& A, hipStream_t st) {
  if (A.parts) {
    attend_shares_kernel<kF16, kCap, kBias, kPage16><<<kShares, 256, 0, st>>>(A);
    join_kernel<kF16><<<kJoinGrid, kJoinThreads, 0, st>>>(A);
  } else {
    attend_tiles_kernel<kF16, kCap, kBias, kPage16><<<(unsigned)(A.n_places * A.p.n_kv_heads), 256, 0, st>>>(A);
  }
}
template <bool kF16, bool kCap, bool kBias>
void launch_pages(const AttendLaunch& A, hipStream_t st) {
  const rkv_pages& p = A.p;
  const bool near = p.k_page < kStrideEnd && p.v_page < kStrideEnd && p.k_slot >= kHeadDim && p.v_slot >= kHeadDim;
  if (p.page_size % 16 == 0 && near) launch_kernels<kF16, kCap, kBias, true>(A, st);
  else launch_kernels<kF16, kCap, kBias, false>(A, st);
}
template <bool kF16>
void launch_type(const AttendLaunch& A, hipStream_t st) {
  if (A.a.softcap > 0.f) {
    if (A.a.slopes) launch_pages<kF16, true, true>(A, st);
    else launch_pages<kF16, true, false>(A, st);
  } else {
    if (A.a.slopes) launch_pages<kF16, false, true>(A, st);
    else launch_pages<kF16, false, false>(A, st);
  }
}

}  // namespace

int launch_attend(const AttendLaunch& A, void* stream) {
  if (A.p.dtype == RKV_F16) launch_type<true>(A, reinterpret_cast<hipStream_t>(stream));
  else launch_type<false>(A, reinterpret_cast<hipStream_t>(stream));
  return (int)hipGetLastError();
}

}  // namespace rkv
