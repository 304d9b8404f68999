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
// One pass with a running maximum m (log2 units), sum l and output O^T per row, rescaled only when a maximum outgrows the
// reference by more than 8 (factors of exp2(8) at most in P, which has the exponent range for it).
#include <hip/hip_runtime.h>

#include "lds_dma.h"
#include "rkv_internal.h"

namespace rkv {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

constexpr int kRows = 128;                 // rows of a workgroup, 32 a wave
constexpr int kKeys = 64;                  // keys of a streamed tile
constexpr int kTileBytes = kKeys * kHeadDim * 2;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kGrow = 8.f;               // log2 units a maximum may outgrow the reference by

__device__ __align__(256) uint32_t zero_row[kHeadDim / 2];   // what a slot outside the visible ones reads as

__device__ __forceinline__ int div_by(int n, FastDiv d) { return (int)(__umulhi((uint32_t)n << 1, d.mul) >> d.shift); }

template <bool kF16>
__device__ __forceinline__ f32x16 mma32(u32x4 a, u32x4 b, f32x16 c) {
  if constexpr (kF16) return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
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
// All of this wave's DMA is in and its LDS reads are done, then the workgroup's.
__device__ __forceinline__ void tile_sync() {
  wait_vmcnt<0>();
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt 0
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}
__device__ __forceinline__ float max_halves(float x) { return fmaxf(x, __shfl_xor(x, 32)); }
__device__ __forceinline__ int wave_min(int x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x = min(x, __shfl_xor(x, o));
  return x;
}
__device__ __forceinline__ int wave_max(int x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x = max(x, __shfl_xor(x, o));
  return x;
}

// First row of sequence s among all, cut to the call's rows.
__device__ __forceinline__ int first_row(const rkv_attend& a, int s) {
  return a.cu_q ? min(max(a.cu_q[s], 0), a.n_rows) : min(s, a.n_rows);
}

// Row tiles are numbered with room for a part-filled one per sequence: sequence s starts at floor(first_row G / 128) + s, which
// ascends and leaves each sequence ceil(rows / 128) numbers, so no list of tiles has to be built.  The sequence of a
// tile: 64-way bisection by one wave.
__device__ __forceinline__ int tile_start(const AttendLaunch& A, int s) { return first_row(A.a, s) * A.group / kRows + s; }
__device__ __forceinline__ int tile_sequence(const AttendLaunch& A, int tile) {
  int lo = 0, n = A.a.n_seqs;
  while (n > 1) {
    const int step = (n + 63) / 64, at = (int)(threadIdx.x & 63) * step;
    const uint64_t in = __ballot(at < n && tile_start(A, lo + at) <= tile);
    const int k = max(0, (int)__popcll(in) - 1) * step;
    lo += k;
    n = min(step, n - k);
  }
  return lo;
}

// kExtra: capped scores or a bias by distance.
template <bool kF16, bool kExtra>
__global__ __launch_bounds__(256, 2) void attend_kernel(const AttendLaunch A) {
  __shared__ __align__(1024) unsigned char smem[4 * kTileBytes];   // [buffer][K, V]
  __shared__ int sLo[4], sHi[4];
  const rkv_attend& a = A.a;
  const rkv_pages& p = A.p;
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 31, half = lane >> 5;
  const int h = blockIdx.x % p.n_kv_heads;
  const int tile = A.n_tiles - 1 - blockIdx.x / p.n_kv_heads;   // a causal prompt's longest rows first
  const int seq = __builtin_amdgcn_readfirstlane(tile_sequence(A, tile));
  const int row0 = first_row(a, seq), n_q = (a.cu_q ? first_row(a, seq + 1) : min(seq + 1, a.n_rows)) - row0;
  const int r0 = (tile - tile_start(A, seq)) * kRows, n_rows = n_q * A.group;
  if (r0 < 0 || r0 >= n_rows) return;
  const int n_kv = min(max(a.lens[seq], 0), a.max_pages * p.page_size);

  // this lane's row (rows behind the last repeat it) and the slots it sees
  const int r = min(r0 + 32 * wv + col, n_rows - 1);
  const int t = div_by(r, A.by_group), hq = h * A.group + r - t * A.group;
  const int64_t row = row0 + t;
  const int pos = n_kv - n_q + t;
  int hi = n_kv;
  if (a.causal) hi = min(n_kv, max(pos + 1, a.prefix_lens ? a.prefix_lens[seq] : 0));
  int lo = a.window ? max(0, pos - a.window + 1) : 0;
  if (a.first_keys) lo = max(lo, a.first_keys[row]);
  if (lo >= hi) {
    lo = 0x7fffffff;
    hi = 0;
  }
  const int w_lo = wave_min(lo), w_hi = wave_max(hi);      // slots some row of the wave sees
  const int all_lo = wave_max(lo), all_hi = wave_min(hi);  // and that every row sees
  if (lane == 0) {
    sLo[wv] = w_lo;
    sHi[wv] = w_hi;
  }
  __syncthreads();
  const int b_lo = min(min(sLo[0], sLo[1]), min(sLo[2], sLo[3])), b_hi = max(max(sHi[0], sHi[1]), max(sHi[2], sHi[3]));
  const int t0 = b_hi > b_lo ? b_lo / kKeys : 0, t1 = b_hi > b_lo ? (b_hi + kKeys - 1) / kKeys : 0;

  u32x4 q[8];
  const uint16_t* qrow = static_cast<const uint16_t*>(a.q) + row * a.q_token + hq * a.q_head;
#pragma unroll
  for (int s = 0; s < 8; ++s) q[s] = *reinterpret_cast<const u32x4*>(qrow + 16 * s + 8 * half);

  // The four rows this lane fetches of a tile: 16 wv + 4 j + lane / 16, 16 bytes of each.  K rows lie in LDS with chunk c at
  // c ^ (row % 16), V rows with c at c ^ 4 (row % 4): the reads below then touch every bank alike.
  const uint32_t lds = lds_addr(smem);
  const int32_t* table = a.table + seq * a.table_stride;
  const char* kp = reinterpret_cast<const char*>(static_cast<const uint16_t*>(p.k) + h * p.k_head);
  const char* vp = reinterpret_cast<const char*>(static_cast<const uint16_t*>(p.v) + h * p.v_head);
  const int fr = lane >> 4;
  int page[4], at[4];
  auto find = [&](int tl) __attribute__((always_inline)) {   // pages of tile tl; -1: not visible, or not in the pool
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int key = tl * kKeys + 16 * wv + 4 * j + fr;
      const bool in = key >= b_lo && key < b_hi;
      const int c = div_by(in ? key : 0, A.by_page);
      at[j] = key - c * p.page_size;
      page[j] = in ? table[c] : -1;
    }
  };
  auto fetch = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bool in = (uint32_t)page[j] < (uint32_t)p.n_pages;
      const uint32_t to = lds + buf * 2 * kTileBytes + (16 * wv + 4 * j) * 256;
      const char* k = in ? kp + 2 * (page[j] * p.k_page + at[j] * p.k_slot) : reinterpret_cast<const char*>(zero_row);
      const char* v = in ? vp + 2 * (page[j] * p.v_page + at[j] * p.v_slot) : reinterpret_cast<const char*>(zero_row);
      dma16(k + 16 * ((lane & 15) ^ (4 * j + fr)), to);
      dma16(v + 16 * ((lane & 15) ^ (4 * fr)), to + kTileBytes);
    }
  };

  f32x16 o[4] = {};
  float m = -__builtin_inff(), l = 0.f;
  const float sl2 = a.scale * kLog2e;
  const float slope = kExtra && a.slopes ? a.slopes[hq] * kLog2e : 0.f;
  const float cap = a.softcap, in_cap = kExtra && cap > 0.f ? 2.f * a.scale / cap * kLog2e : 0.f;
  const uint32_t k_lane = col * 256 + ((col & 15) ^ half) * 16;
  // V^T: lane reads 4 columns of key 4 half + (lane % 16) / 4 (+ 8), chunk 4 dt + 2 ((lane / 16) % 2) + (lane % 4) / 2
  const int v_key = 4 * half + ((lane & 15) >> 2);
  const uint32_t v_lane = v_key * 256 + ((2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ (4 * (v_key & 3))) * 16 + (lane & 1) * 8;

  if (t0 < t1) {
    find(t0);
    fetch(0);
    if (t0 + 1 < t1) find(t0 + 1);
  }
  for (int tl = t0; tl < t1; ++tl) {
    const int buf = (tl - t0) & 1;
    tile_sync();
    if (tl + 1 < t1) {
      fetch(buf ^ 1);
      if (tl + 2 < t1) find(tl + 2);
    }
    const int key0 = tl * kKeys;
    if (key0 + kKeys <= w_lo || key0 >= w_hi) continue;   // the other waves' rows see it
    const uint32_t kb = lds + buf * 2 * kTileBytes, vb = kb + kTileBytes;
    f32x16 s[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      s[u] = f32x16{};
#pragma unroll
      for (int st = 0; st < 8; ++st) s[u] = mma32<kF16>(lds_read16(kb + u * 8192 + (k_lane ^ (32 * st))), q[st], s[u]);
    }
    // key of s[u][i]: key0 + 32 u + 8 (i / 4) + 4 half + i % 4
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        float x = s[u][i];
        if constexpr (kExtra) {
          // cap tanh(x / cap) = cap (1 - 2 / (1 + exp(2 x / cap)))
          if (in_cap != 0.f) x = cap * kLog2e * (1.f - 2.f * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x * in_cap)));
          else x *= sl2;
          x -= slope * fabsf((float)(pos - (key0 + 32 * u + 8 * (i >> 2) + 4 * half + (i & 3))));
        } else {
          x *= sl2;
        }
        s[u][i] = x;
      }
    if (key0 < all_lo || key0 + kKeys > all_hi) {
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int key = key0 + 32 * u + 8 * (i >> 2) + 4 * half + (i & 3);
          if (key < lo || key >= hi) s[u][i] = -__builtin_inff();
        }
    }
    float top = s[0][0];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, s[u][i]);
    top = max_halves(top);
    if (__any(top > m + kGrow)) {
      const float m2 = fmaxf(m, top), f = m2 > m ? __builtin_amdgcn_exp2f(m - m2) : 1.f;
      m = m2;
      l *= f;
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] *= f;
    }
    const float ref = m == -__builtin_inff() ? 0.f : m;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[u][i] = __builtin_amdgcn_exp2f(s[u][i] - ref);
        l += s[u][i];
      }
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {   // 16 keys each
      u32x4 pr;
#pragma unroll
      for (int i = 0; i < 4; ++i) pr[i] = pack<kF16>(s[ks >> 1][8 * (ks & 1) + 2 * i], s[ks >> 1][8 * (ks & 1) + 2 * i + 1]);
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        const u32x2 v0 = lds_read_tr(vb + ks * 4096 + (v_lane ^ (64 * d)));
        const u32x2 v1 = lds_read_tr(vb + ks * 4096 + 2048 + (v_lane ^ (64 * d)));
        o[d] = mma32<kF16>(u32x4{v0[0], v0[1], v1[0], v1[1]}, pr, o[d]);
      }
    }
  }

  l += __shfl_xor(l, 32);
  if (r0 + 32 * wv + col >= n_rows) return;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  uint16_t* out = static_cast<uint16_t*>(a.out) + row * a.out_token + hq * a.out_head + 4 * half;
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<u32x2*>(out + 32 * d + 8 * i) =
          u32x2{pack<kF16>(o[d][4 * i] * inv, o[d][4 * i + 1] * inv), pack<kF16>(o[d][4 * i + 2] * inv, o[d][4 * i + 3] * inv)};
  if (a.lse && half == 0) a.lse[row * a.n_q_heads + hq] = l == 0.f ? -__builtin_inff() : m / kLog2e + logf(l);
}

template <bool kF16>
void launch_type(const AttendLaunch& A, hipStream_t st) {
  const unsigned grid = (unsigned)(A.n_tiles * A.p.n_kv_heads);
  if (A.a.softcap > 0.f || A.a.slopes) attend_kernel<kF16, true><<<grid, 256, 0, st>>>(A);
  else attend_kernel<kF16, false><<<grid, 256, 0, st>>>(A);
}

}  // namespace

int launch_attend(const AttendLaunch& A0, void* stream) {
  AttendLaunch A = A0;
  A.n_tiles = (int)((int64_t)A.a.n_rows * A.group / kRows) + A.a.n_seqs;
  if (A.p.dtype == RKV_F16) launch_type<true>(A, reinterpret_cast<hipStream_t>(stream));
  else launch_type<false>(A, reinterpret_cast<hipStream_t>(stream));
  return (int)hipGetLastError();
}

}  // namespace rkv
