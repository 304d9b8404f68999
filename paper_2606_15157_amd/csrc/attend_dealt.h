// Attention over pages for pools of 8-bit codes and for sequences that share prefixes: how row tiles are dealt out.
//
// Row tiles of more than 16 rows (prompts, chunks, the rows of a group over its prefix) need a workgroup: their keys go through LDS and
// their products fill the matrix pipes.  Tiles of fewer (decode steps, drafts) are a stream of keys with little to do: a wave takes them by
// itself, from memory to registers, waits for no other, and does not stop at the end of an item for three more.  So a launch's
// workgroups are divided, by the work on either side: some take equal shares of the wide tiles' key tiles, the waves of the others equal
// shares of the narrow ones'.  A workgroup that went from one sequence of a few key tiles to the next lost 5 us on each (a table, then
// keys, then the sums of four waves, each waited for): with 64 requests of 64 keys to a prefix, 5.4 us a workgroup.
//
// Parts of a tile that several shares have go to the workspace, and a join by row adds them up in the order of the keys, the prefix's
// first: which these are is in a record for each row and head.
#pragma once

#include "attend_rows.h"

namespace rkv {
namespace {

constexpr int kDealt = kAttendDealt;
// Record of a row and head: m, l (relative to what, and the sum) if one share has all of it, then the number of parts (0: one share has
// all) and these bits, then the first part's share and from bit 16 the row among its tile's.
constexpr int kParts = 4095, kHasPrefix = 1 << 16, kFewRows = 1 << 17;

// What an item costs besides its key tiles, in key tiles: it begins with a table, then keys, each waited for, and ends with stores (some 5 us
// of a workgroup where a key tile takes 1.5, 9 us of a wave where one takes 3 to 4).  Shares of many tiles count it, as units before the first
// one; where there is little to do for all, shares are as small as can be.
constexpr int kItem = 3;

// The list of row tiles that every workgroup makes: those of the groups over their prefixes, then those of the sequences.
struct Deal {
  int32_t row0[kDealt + 2];       // first row of each group and behind the last, then of each sequence
  int32_t slots[kDealt];          // of each prefix, then of each sequence
  int32_t wide[kDealt + 1];       // units of a head before row tile i, of those with more than 16 rows
  int32_t few[kDealt + 1];        // and of the others
  uint16_t seq[kDealt];           // group or sequence of row tile i, and kPrefixed
  int32_t sums[4][kDealt / 64];
  int32_t early;                  // whether some sequence has rows before its last prefix slot
};
constexpr int kPrefixed = 1 << 15;

// Of a head: key tiles and row tiles of either kind; workgroups (of an XCD's) for the wide ones; units besides the key tiles that an item counts for.
struct Totals {
  int wide, few, wide_items, few_items, n_wide, wide_extra, few_extra;
};
// Workgroups (of the kShares / 8 of an XCD) for the wide tiles, so that either side ends at the same time.  By time stamps, us: a wide tile's 64 keys
// take a workgroup 1.8, in 8 bits 2.1 (their way into LDS is by registers); those of a narrow one take a wave 5 to 6, or 3 in 8 bits, as long
// as the chip's memory does not bound them, and a narrow item 6 to 8 besides; a workgroup has four waves.  The weights below, 1.6 and 2.3, are from
// before 8-bit codes went to LDS beside the products, and no rule for all shapes: with 2.0 for 2.3 128 requests in eight groups take 196 us for
// 215, but all in one 118 for 115, and 64 in one 47 for 43.5.
template <Pool kPool>
__device__ __forceinline__ int wide_workgroups(const Totals& all) {
  constexpr int kMost = kShares / 8;
  if (!all.wide) return 0;
  if (!all.few) return kMost;
  const float wide = (in_codes(kPool) ? 2.3f : 1.6f) * (float)(all.wide + kItem * all.wide_items);
  const float few = (in_codes(kPool) ? 0.75f : 1.4f) * (float)all.few + (in_codes(kPool) ? 1.6f : 2.f) * (float)all.few_items;
  return min(max((int)(wide / (wide + few) * kMost + 0.5f), 1), kMost - 1);
}
__device__ __forceinline__ int extra_units(int tiles, int items, int heads, int shares) {
  return ((int64_t)tiles + kItem * items) * heads >= (int64_t)2 * kItem * shares ? kItem : 0;
}
// Fills the list; the units of a head, fewer than 2^31 (the host lets no other call here).
template <Pool kPool, bool kShared>
__device__ __forceinline__ Totals deal(const AttendLaunch& A, Deal& L, int groups, int seqs) {
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, own0 = groups ? groups + 1 : 0;
  int first_prefixed = 0, end_prefixed = 0;
  bool early = false;
  if constexpr (kShared) {
    first_prefixed = A.g.cu_seqs[0];
    end_prefixed = A.g.cu_seqs[A.g.n_groups];
  }
  // What a thread loads of a group and of a sequence it loads at once: one wait, and one more for the groups' rows.
  const int32_t* cu = A.a.cu_q;
  for (int s = tid; s <= max(groups, A.a.n_seqs); s += 256) {
    const int last = A.a.n_seqs - 1;
    const int c0 = cu ? cu[min(s, last + 1)] : s, c1 = cu ? cu[min(s, last) + 1] : s + 1, n_kv = last >= 0 ? slots_of(A, min(s, last)) : 0;
    if constexpr (kShared) {
      if (s <= groups && groups) {
        const int member = A.g.cu_seqs[s], slots = slots_of<kShared>(A, min(s, groups - 1), true);
        L.row0[s] = min(max(cu ? cu[min(max(member, 0), A.a.n_seqs)] : min(max(member, 0), A.a.n_seqs), 0), A.a.n_rows);
        if (s < groups) L.slots[s] = slots;
      }
      early |= groups && s <= last && A.a.causal && c1 - c0 > n_kv + 1;
    }
    if (s <= seqs && seqs) {
      L.row0[own0 + s] = min(max(c0, 0), A.a.n_rows);
      if (s < seqs) L.slots[groups + s] = n_kv;
    }
  }
  if constexpr (kShared) {
    const int some = __syncthreads_or(early);
    if (tid == 0) L.early = some;
  } else {
    __syncthreads();
  }
  // A tile a thread: 256 at a time, as many times as there are tiles.
  int cost[kDealt / 256], x_wide[kDealt / 256], x_few[kDealt / 256], i_wide[kDealt / 256], i_few[kDealt / 256];
  bool narrow[kDealt / 256];
#pragma unroll
  for (int i = 0; i < kDealt / 256; ++i) {
    const int tile = 256 * i + tid;
    cost[i] = 0;
    narrow[i] = false;
    if (256 * i < A.n_tiles && tile < A.n_tiles) {
      const bool over = kShared && tile < A.n_group_tiles;
      const int at = over || !kShared ? tile : tile - A.n_group_tiles, base = over ? 0 : own0;
      int lo = 0, hi = over ? groups : seqs;
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (tile_start(A, L.row0[base + mid], mid) <= at) lo = mid;
        else hi = mid;
      }
      L.seq[tile] = (uint16_t)(lo | (!over && lo >= first_prefixed && lo < end_prefixed ? kPrefixed : 0));
      const int row0 = L.row0[base + lo], n_q = L.row0[base + lo + 1] - row0, r0 = (at - tile_start(A, row0, lo)) * kRows;
      if (r0 >= 0 && r0 < n_q * A.group) {
        int t0, t1;
        tile_span<kShared>(A, lo, r0, n_q, L.slots[over ? lo : groups + lo], over, t0, t1);
        cost[i] = max(1, t1 - t0);   // rows that see nothing are written too
        narrow[i] = n_q * A.group - r0 <= 16;
      }
    }
    x_wide[i] = narrow[i] ? 0 : cost[i];
    x_few[i] = narrow[i] ? cost[i] : 0;
    if (256 * i < A.n_tiles) {
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(x_wide[i], o), z = __shfl_up(x_few[i], o);
        if (lane >= o) {
          x_wide[i] += y;
          x_few[i] += z;
        }
      }
    }
    const uint64_t few = __ballot(narrow[i]), wide = __ballot(cost[i] && !narrow[i]), below = ((uint64_t)1 << lane) - 1;
    i_wide[i] = (int)__popcll(wide & below);      // row tiles before this one
    i_few[i] = (int)__popcll(few & below);
    if (lane == 63) {
      L.sums[0][4 * i + wv] = x_wide[i];
      L.sums[1][4 * i + wv] = x_few[i];
      L.sums[2][4 * i + wv] = (int)__popcll(wide);
      L.sums[3][4 * i + wv] = (int)__popcll(few);
    }
  }
  __syncthreads();
  Totals all = {};
#pragma unroll
  for (int i = 0; i < kDealt / 256; ++i) {
    if (256 * i >= A.n_tiles) break;
    x_wide[i] += all.wide - (narrow[i] ? 0 : cost[i]);
    x_few[i] += all.few - (narrow[i] ? cost[i] : 0);
    i_wide[i] += all.wide_items;
    i_few[i] += all.few_items;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int wide = L.sums[0][4 * i + j], few = L.sums[1][4 * i + j], wide_items = L.sums[2][4 * i + j], few_items = L.sums[3][4 * i + j];
      if (j < wv) {
        x_wide[i] += wide;
        x_few[i] += few;
        i_wide[i] += wide_items;
        i_few[i] += few_items;
      }
      all.wide += wide;
      all.few += few;
      all.wide_items += wide_items;
      all.few_items += few_items;
    }
  }
  all.wide = uniform(all.wide);
  all.few = uniform(all.few);
  all.wide_items = uniform(all.wide_items);
  all.few_items = uniform(all.few_items);
  all.n_wide = uniform(wide_workgroups<kPool>(all));
  all.wide_extra = extra_units(all.wide, all.wide_items, A.p.n_kv_heads, 8 * all.n_wide);
  all.few_extra = extra_units(all.few, all.few_items, A.p.n_kv_heads, 4 * (kShares - 8 * all.n_wide));
#pragma unroll
  for (int i = 0; i < kDealt / 256; ++i) {
    if (256 * i >= A.n_tiles) break;
    L.wide[256 * i + tid] = x_wide[i] + all.wide_extra * i_wide[i];
    L.few[256 * i + tid] = x_few[i] + all.few_extra * i_few[i];
  }
  __syncthreads();      // what a thread of no tile wrote is behind the last one's
  all.wide += all.wide_extra * all.wide_items;      // units from here on
  all.few += all.few_extra * all.few_items;
  if (tid == 0) {
    L.wide[A.n_tiles] = all.wide;
    L.few[A.n_tiles] = all.few;
  }
  __syncthreads();
  return all;
}

// a / b for a >= 0 and b > 0; two 64-bit divisions are a third of a microsecond.
__device__ __forceinline__ int64_t divide(int64_t a, int64_t b) {
  if ((a | b) >> 32 == 0) return (uint32_t)a / (uint32_t)b;
  return a / b;
}

// How units are shared out.  Of a CU's two workgroups the one that came first is served first: with equal shares of 512 tokens after 32768 the
// first ones took 257 us and the others 322, of four sequences of 131072 146 and 171.  So shares go by weights, 4 to 3, where even the smaller ones
// hold `least` units; else all hold as many as need be for that.
struct Cut {
  int64_t total, share;      // share: of every one, or 0
  int n, n_first, first, second;      // shares of an XCD, those of its CUs' first workgroups, and weights
  __device__ __forceinline__ int weight() const { return n_first * first + (n - n_first) * second; }      // of an XCD
  __device__ __forceinline__ void set(int64_t units, int shares, int of_first, int w_first, int w_second, int least) {
    total = units;
    n = shares;
    n_first = of_first;
    first = w_first;
    second = w_second;
    const double smallest = (double)total * second / (8 * weight());
    share = smallest >= least + 1 ? 0 : max((int64_t)least, divide(total + 8 * n - 1, 8 * n));
  }
  // The first unit of share w.
  __device__ __forceinline__ int64_t begin(int w) const {
    if (share) return min(total, w * share);
    if (w >= 8 * n) return total;
    const int x = w / n, j = w - x * n;
    const int before = x * weight() + (j < n_first ? j * first : n_first * first + (j - n_first) * second);
    return (int64_t)((double)total * before / (8 * weight()));
  }
  // The share that unit p belongs to.
  __device__ __forceinline__ int of(int64_t p) const {
    if (share) return (int)divide(p, share);
    const int at = (int)((double)p * (8 * weight()) / (double)total), x = min(at / weight(), 7), r = at - x * weight();
    int w = x * n + min(r < n_first * first ? r / first : n_first + (r - n_first * first) / second, n - 1);
    while (begin(w) > p) --w;
    while (begin(w + 1) <= p) ++w;
    return w;
  }
};

// Shares of the row tiles' units, in the order (head, row tile, key tile), are consecutive.  Workgroup b runs on XCD b % 8 and
// takes shares that follow those of the XCD before, so that the tiles of a head, which read the same keys, meet in one L2.
template <bool kF16, bool kCap, bool kBias, Pool kPool, bool kShared>
__global__ __launch_bounds__(256, 2) void attend_dealt_kernel(const AttendLaunch A) {
  __shared__ __align__(1024) unsigned char smem[4 * kTileBytes];
  __shared__ Bounds bounds;
  __shared__ Deal L;
  const int groups = kShared && A.stage != kOverOwn ? A.g.n_groups : 0, seqs = kShared && A.stage == kOverPrefix ? 0 : A.a.n_seqs;
  const Totals all = deal<kPool, kShared>(A, L, groups, seqs);
  const int xcd = blockIdx.x % 8, at_xcd = blockIdx.x / 8, n_wide = all.n_wide;
  // This workgroup's shares, or this wave's.
  auto take = [&](auto few, const int32_t* before, int units, int extra, int w, const Cut& cut) __attribute__((always_inline)) {
    constexpr bool kFew = decltype(few)::value;
    const int tid = kFew ? threadIdx.x & 63 : threadIdx.x;
    int64_t pos = cut.begin(w);
    const int64_t end = cut.begin(w + 1);
    while (pos < end) {
      const int h = uniform((int)divide(pos, units)), rem = uniform((int)(pos - (int64_t)h * units));
      int lo = 0, hi = A.n_tiles;
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (before[mid] <= rem) lo = mid;
        else hi = mid;
      }
      const int tile = uniform(lo), named = uniform(L.seq[tile]), seq = named & ~kPrefixed;
      const bool over = kShared && tile < A.n_group_tiles;
      const int v = over || !groups ? seq : groups + 1 + seq, at = over || !kShared ? tile : tile - A.n_group_tiles;
      const int x0 = rem - uniform(before[tile]), count = uniform(before[tile + 1]) - uniform(before[tile]);
      const int x = (int)min((int64_t)(count - x0), end - pos);
      const int u0 = max(0, x0 - extra), n = max(0, x0 + x - extra) - u0;      // key tiles
      pos += x;
      if (n == 0) continue;      // the next share begins it
      const int row0 = uniform(L.row0[v]), n_q = uniform(L.row0[v + 1]) - row0, r0 = (at - tile_start(A, row0, seq)) * kRows;
      float* part = nullptr;
      int word = 0;
      if (n < count - extra) {
        part = kFew ? few_slot(A, 2 * w + (u0 == 0)) : part_slot(A, 2 * w + (u0 == 0));
        if (u0 == 0) word = (cut.of(pos - x - x0 + count - 1) - w + 1) | (kFew ? kFewRows : 0);
      }
      if (u0 == 0) {
        if (named & kPrefixed) word |= kHasPrefix;
        for (int r = r0 + tid; r < min(n_q * A.group, r0 + kRows); r += kFew ? 64 : 256) {
          const int t = div_by(r, A.by_group), hq = h * A.group + r - t * A.group;
          reinterpret_cast<i32x2*>(sums_scale(A, row0 + t, hq, A.stage == kBoth && !over))[1] = i32x2{word, w | (r - r0) << 16};
        }
      }
      const int n_kv = uniform(L.slots[over ? seq : groups + seq]);
      attend_rows<kF16, kCap, kBias, kPool, kShared, kFew, kFew>(A, smem, bounds, seq, row0, n_q, n_kv, r0, h, u0, n, part, over, kShared && L.early);
      if constexpr (!kFew) lds_sync();   // the memory that rows left by is the next tiles'
    }
  };
  constexpr int kFirst = kShares / 16;      // workgroups of an XCD that are their CU's first
  Cut cut;
  if (at_xcd < n_wide) {
    cut.set((int64_t)all.wide * A.p.n_kv_heads, n_wide, min(n_wide, kFirst), 4, 3, A.least + all.wide_extra);
    take(Flag<false>{}, L.wide, all.wide, all.wide_extra, xcd * n_wide + at_xcd, cut);
  } else {
    const int n_few = kShares / 8 - n_wide;
    cut.set((int64_t)all.few * A.p.n_kv_heads, 4 * n_few, 4 * max(0, kFirst - n_wide), 4, 3, 1 + all.few_extra);
    take(Flag<true>{}, L.few, all.few, all.few_extra, 4 * (xcd * n_few + at_xcd - n_wide) + uniform(threadIdx.x >> 6), cut);
  }
}

// Rows of which several shares have parts, by the records of each row and head; with kBoth all rows, whose sums over the prefix
// and over the own slots meet here.  32 lanes hold the 128 values of a row, 8 rows a workgroup, or fewer whose parts several groups of lanes
// take in turn and that meet in LDS.
template <bool kF16, bool kShared>
__global__ __launch_bounds__(kJoinThreads) void join_rows_kernel(const AttendLaunch A) {
  __shared__ f32x4 sO[8][32];
  __shared__ float sM[8], sL[8];
  const rkv_attend& a = A.a;
  const int tid = threadIdx.x, grp = tid >> 5, c = tid & 31;
  const bool both = kShared && A.stage == kBoth, over_prefix = kShared && A.stage == kOverPrefix;
  const int begin = first_row<kShared>(A, 0, over_prefix), stop = first_row<kShared>(A, over_prefix ? A.g.n_groups : a.n_seqs, over_prefix);
  const int64_t first = (int64_t)begin * a.n_q_heads, total = (int64_t)stop * a.n_q_heads;      // rows of no sequence are not touched
  int most = 8;
  while (most > 1 && (total - first + most - 1) / most < kJoinGrid) most >>= 1;
  const int each = 8 / most, i = grp / each, g = grp - i * each;
  for (int64_t task = first + (int64_t)blockIdx.x * most; task < total; task += (int64_t)kJoinGrid * most) {
    const int64_t id = task + i;
    const bool in = id < total;
    const int64_t row = (in ? id : task) / a.n_q_heads;
    const int hq = (int)((in ? id : task) - row * a.n_q_heads);
    const f32x4 own = *reinterpret_cast<const f32x4*>(sums_scale(A, row, hq, both));
    f32x4 pre = {0.f, 0.f, 0.f, 0.f};
    if (both) pre = *reinterpret_cast<const f32x4*>(sums_scale(A, row, hq));      // undefined without a prefix
    const int own_word = __float_as_int(own[2]), own_parts = own_word & kParts;
    const bool with_prefix = both && (own_word & kHasPrefix);
    const int pre_word = __float_as_int(pre[2]), pre_parts = pre_word & kParts;
    const int n_pre = with_prefix ? max(1, pre_parts) : 0, n = n_pre + (both ? max(1, own_parts) : own_parts);   // alone, a whole row is finished
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
    for (int j0 = g; j0 < n; j0 += 4 * each) {   // four parts in flight
      f32x2 ml[4];
      f32x4 v[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int jj = min(j0 + j * each, n - 1);
        const bool over = jj < n_pre;
        const int k = over ? jj : jj - n_pre, where = __float_as_int(over ? pre[3] : own[3]), word = over ? pre_word : own_word;
        const float *from_o = sums_row(A, row, hq, both && !over), *from_m = sums_scale(A, row, hq, both && !over);
        if (word & kParts) {      // cut to the workspace, whatever cu_q and cu_seqs hold
          const bool few = word & kFewRows;
          const int share = min((where & 0xffff) + k, (few ? 4 : 1) * kShares - 1), rows = few ? A.few_rows : A.slot_rows, at = min((int)((uint32_t)where >> 16), rows - 1);
          const float* from = few ? few_slot(A, k ? 2 * share : 2 * share + 1) : part_slot(A, k ? 2 * share : 2 * share + 1);
          from_o = from + at * kHeadDim;
          from_m = from + rows * kHeadDim + 2 * at;
        }
        ml[j] = *reinterpret_cast<const f32x2*>(from_m);
        v[j] = *reinterpret_cast<const f32x4*>(from_o + 4 * c);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (j0 + j * each < n) add(ml[j][0], ml[j][1], v[j]);
    }
    if (each > 1) {
      __syncthreads();   // sO is free
      sO[grp][c] = acc;
      if (c == 0) {
        sM[grp] = m;
        sL[grp] = l;
      }
      __syncthreads();
      if (g == 0)
        for (int x = 1; x < each; ++x) add(sM[grp + x], sL[grp + x], sO[grp + x][c]);
    }
    if (!in || g || !n) continue;
    if (over_prefix) {
      *reinterpret_cast<f32x4*>(sums_row(A, row, hq) + 4 * c) = acc;
      if (c == 0) *reinterpret_cast<f32x2*>(sums_scale(A, row, hq)) = f32x2{m, l};
      continue;
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    uint16_t* out = static_cast<uint16_t*>(a.out) + row * a.out_token + hq * a.out_head + 4 * c;
    *reinterpret_cast<u32x2*>(out) = u32x2{pack<kF16>(acc[0] * inv, acc[1] * inv), pack<kF16>(acc[2] * inv, acc[3] * inv)};
    if (a.lse && c == 0) a.lse[row * a.n_q_heads + hq] = row_lse(m, l);
  }
}

template <bool kF16, bool kCap, bool kBias, Pool kPool, bool kShared>
void launch_dealt(const AttendLaunch& A, hipStream_t st) {
  if (A.parts) {
    attend_dealt_kernel<kF16, kCap, kBias, kPool, kShared><<<kShares, 256, 0, st>>>(A);
    join_rows_kernel<kF16, kShared><<<kJoinGrid, kJoinThreads, 0, st>>>(A);
  } else {
    attend_tiles_kernel<kF16, kCap, kBias, kPool, kShared><<<(unsigned)(A.n_places * A.p.n_kv_heads), 256, 0, st>>>(A);
  }
}

}  // namespace
}  // namespace rkv
