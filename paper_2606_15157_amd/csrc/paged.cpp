// Host side of the paged caches: argument checks and launches of rkv_pages_* and, for pools of 8-bit codes, rkv_qpages_*.
#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <array>
#include <cmath>
#include <initializer_list>

#include "paged.h"

namespace {

constexpr int64_t kIntEnd = int64_t(1) << 31;
constexpr int64_t kGridEnd = int64_t(1) << 24;   // workgroups of 256 threads: HIP takes fewer than 2^32 threads in x

int launched(int err) {
  if (err) return rkv::fail(RKV_ERR_HIP, std::string("kernel launch failed: ") + hipGetErrorString((hipError_t)err));
  return RKV_OK;
}

// A 16-byte aligned pointer and strides (elements) of whole 16-byte pieces, `piece` elements each.
int check_layout(const char* what, const void* ptr, std::initializer_list<int64_t> strides, int piece = 8) {
  for (int64_t s : strides)
    if (s < 0) return rkv::fail(RKV_ERR_INVALID_ARG, std::string(what) + ": negative stride");
  if ((uintptr_t)ptr % 16) return rkv::fail(RKV_ERR_UNSUPPORTED, std::string(what) + " must be 16-byte aligned");
  for (int64_t s : strides)
    if (s % piece)
      return rkv::fail(RKV_ERR_UNSUPPORTED, std::string(what) + ": strides must be multiples of " + std::to_string(piece) + " elements");
  return RKV_OK;
}

// Whether rows of `extent` elements, at sum_i index_i stride_i for index_i < count_i, are told apart by their dimensions: taken by
// stride, each is at least the extent of the smaller ones.  So are those of every slice and permutation of a dense tensor.
struct Dim {
  int64_t stride, count;
};
template <size_t kDims>
bool rows_nest(std::array<Dim, kDims> dims, __int128 extent = rkv::kHeadDim) {
  std::sort(dims.begin(), dims.end(), [](const Dim& x, const Dim& y) { return x.stride < y.stride; });
  for (const Dim& d : dims) {
    if (d.count <= 1) continue;
    if (d.stride < extent) return false;
    extent += (__int128)d.stride * (d.count - 1);
  }
  return true;
}

// Rows of `extent` elements of `size` bytes from `at` on, told apart by their dimensions as above.
struct Rows {
  const void* at;
  int size;
  __int128 extent;
  std::array<Dim, 3> dims;
};
// Whether a row of x and a row of y may share a byte, from the i-th largest stride of each on, y `apart` elements behind x.  Apart they are
// where all of one lies behind all of the other; else, of slices along one stride that both have, each can only meet the two that
// are less than it away, for a slice is no longer than the stride.  Where both lie in one piece of memory by different strides they count as met.
bool slices_meet(const std::array<Dim, 4>& x, const std::array<Dim, 4>& y, const std::array<__int128, 4>& x_extent, const std::array<__int128, 4>& y_extent, int i,
                 __int128 apart) {
  if (apart >= x_extent[i] || -apart >= y_extent[i]) return false;
  const Dim &dx = x[i], &dy = y[i];
  if (dx.count == 0 || dx.stride != dy.stride) return true;     // rows, or strides that differ
  const __int128 s = dx.stride;
  __int128 d = -apart / s - (-apart % s < 0);                  // rounded down
  for (int k = 0; k < 2; ++k, ++d)
    if (d > -dx.count && d < dy.count && slices_meet(x, y, x_extent, y_extent, i + 1, apart + d * s)) return true;
  return false;
}
__int128 whole(const Rows& r) {
  __int128 extent = r.extent;
  for (const Dim& d : r.dims) extent += (__int128)d.stride * (d.count - 1);
  return extent;
}
bool rows_meet(const Rows& x, const Rows& y) {
  const __int128 apart = ((__int128)(uintptr_t)y.at - (__int128)(uintptr_t)x.at) / x.size;
  if (apart >= whole(x) || -apart >= whole(y)) return false;      // as in most calls
  std::array<Dim, 4> dims[2] = {};           // those of more than one entry, the largest stride first, then {0, 0}
  std::array<__int128, 4> extents[2] = {};   // of what the strides from i on reach
  for (int k = 0; k < 2; ++k) {
    const Rows& r = k ? y : x;
    int n = 0;
    for (const Dim& d : r.dims)
      if (d.count > 1) dims[k][n++] = d;
    std::sort(dims[k].begin(), dims[k].begin() + n, [](const Dim& a, const Dim& b) { return a.stride > b.stride; });
    extents[k].fill(r.extent);
    for (int i = n - 1; i >= 0; --i) extents[k][i] = extents[k][i + 1] + (__int128)dims[k][i].stride * (dims[k][i].count - 1);
  }
  return slices_meet(dims[0], dims[1], extents[0], extents[1], 0, apart);
}

bool rows_same(const Rows& x, const Rows& y) {
  bool same = x.at == y.at;
  for (size_t i = 0; i < x.dims.size(); ++i) same &= x.dims[i].count <= 1 || x.dims[i].stride == y.dims[i].stride;
  return same;
}

template <class Pages>
int check_pool(const Pages* p) {
  if (!p) return rkv::fail(RKV_ERR_INVALID_ARG, "null pages");
  if (!p->k || !p->v) return rkv::fail(RKV_ERR_INVALID_ARG, "null page pool");
  if (p->n_pages < 1 || p->page_size < 1 || p->n_kv_heads < 1)
    return rkv::fail(RKV_ERR_INVALID_ARG, "n_pages, page_size and n_kv_heads must be >= 1");
  if (p->dtype != RKV_BF16 && p->dtype != RKV_F16) return rkv::fail(RKV_ERR_INVALID_ARG, "unknown dtype");
  if (p->head_dim != rkv::kHeadDim) return rkv::fail(RKV_ERR_UNSUPPORTED, "head_dim must be 128");
  if ((int64_t)p->n_pages * p->page_size >= kIntEnd) return rkv::fail(RKV_ERR_UNSUPPORTED, "a pool holds fewer than 2^31 slots");
  return RKV_OK;
}
int check_pages(const rkv_pages* p) {
  if (int st = check_pool(p)) return st;
  if (p->k_slot >= kIntEnd / 16 || p->v_slot >= kIntEnd / 16)
    return rkv::fail(RKV_ERR_UNSUPPORTED, "slots are fewer than 2^27 elements apart");
  if (int st = check_layout("k pages", p->k, {p->k_page, p->k_head, p->k_slot})) return st;
  return check_layout("v pages", p->v, {p->v_page, p->v_head, p->v_slot});
}
int check_pages(const rkv_qpages* p) {
  if (int st = check_pool(p)) return st;
  if (!p->k_scale || !p->v_scale) return rkv::fail(RKV_ERR_INVALID_ARG, "null scales");
  for (int64_t x : {p->ks_page, p->ks_head, p->ks_slot, p->vs_page, p->vs_head, p->vs_slot})
    if (x < 0) return rkv::fail(RKV_ERR_INVALID_ARG, "scales: negative stride");
  if (int st = check_layout("k pages", p->k, {p->k_page, p->k_head, p->k_slot}, 16)) return st;
  return check_layout("v pages", p->v, {p->v_page, p->v_head, p->v_slot}, 16);
}

// The pool as the launches take it.
struct Pool {
  rkv_pages p;
  rkv::Scales ks, vs;
  bool codes;
};
Pool pool_of(const rkv_pages* p) { return {*p, {}, {}, false}; }
Pool pool_of(const rkv_qpages* p) {
  return {{p->k, p->v, p->k_page, p->k_head, p->k_slot, p->v_page, p->v_head, p->v_slot, p->n_pages, p->page_size, p->n_kv_heads, p->head_dim, p->dtype},
          {p->k_scale, p->ks_page, p->ks_head, p->ks_slot},
          {p->v_scale, p->vs_page, p->vs_head, p->vs_slot},
          true};
}

// Row tiles, with one part-filled tile for each sequence.
int64_t full_tiles(const rkv_pages* p, const rkv_attend* a) { return (int64_t)a->n_rows * (a->n_q_heads / p->n_kv_heads) / rkv::kAttendRows; }
int64_t row_tiles(const rkv_pages* p, const rkv_attend* a) { return full_tiles(p, a) + a->n_seqs; }

// Places of attend_tiles_kernel: the sequences, then the numbers of long sequences' tiles.
int64_t places(const rkv_pages* p, const rkv_attend* a) { return a->n_seqs + std::min(2 * full_tiles(p, a), row_tiles(p, a)); }
bool nothing_to_do(const rkv_attend* a) { return a->n_seqs == 0 || a->n_rows == 0; }
bool shared_out(const rkv_pages* p, const rkv_attend* a);
bool dealt(const rkv_pages* p, const rkv_attend* a);

// A call on a pool that has been checked.  split: whether a list of its key tiles is dealt out.
int check_attend(const rkv_pages* p, const rkv_attend* a, bool (*split)(const rkv_pages*, const rkv_attend*)) {
  if (!a) return rkv::fail(RKV_ERR_INVALID_ARG, "null attend");
  if (a->n_seqs < 0 || a->n_rows < 0 || a->max_pages < 0 || a->max_q < 0 || a->max_kv < 0 || a->window < 0 || a->table_stride < 0)
    return rkv::fail(RKV_ERR_INVALID_ARG, "negative size");
  if (a->causal != 0 && a->causal != 1) return rkv::fail(RKV_ERR_INVALID_ARG, "causal must be 0 or 1");
  if (!std::isfinite(a->scale) || !std::isfinite(a->softcap) || a->softcap < 0.f ||
      (a->softcap > 0.f && std::fabs(a->scale) / a->softcap > 1e30f))
    return rkv::fail(RKV_ERR_INVALID_ARG, "scale and softcap must be finite, softcap >= 0 and not below 1e-30 of the scale");
  if (a->softcap > 512.f) return rkv::fail(RKV_ERR_UNSUPPORTED, "softcap above 512");
  if (a->n_q_heads < 1 || a->n_q_heads % p->n_kv_heads)
    return rkv::fail(RKV_ERR_SHAPE, "n_q_heads must be a positive multiple of n_kv_heads");
  if (!rows_nest<2>({{{a->out_token, a->n_rows}, {a->out_head, a->n_q_heads}}}))
    return rkv::fail(RKV_ERR_INVALID_ARG, "out's rows overlap (no stride may be less than the extent of the smaller ones)");
  if (!a->cu_q && a->n_rows != a->n_seqs) return rkv::fail(RKV_ERR_SHAPE, "without cu_q every sequence has one row");
  if (a->table_stride < a->max_pages) return rkv::fail(RKV_ERR_SHAPE, "table_stride is less than max_pages");
  if ((int64_t)a->max_pages * p->page_size >= kIntEnd - 1024)   // key tiles past the end stay below 2^31
    return rkv::fail(RKV_ERR_UNSUPPORTED, "a sequence holds fewer than 2^31 - 1024 slots");
  if ((int64_t)a->n_rows * a->n_q_heads >= kIntEnd / 2) return rkv::fail(RKV_ERR_UNSUPPORTED, "n_rows * n_q_heads must be below 2^30");
  if (!nothing_to_do(a) && !split(p, a) && places(p, a) * p->n_kv_heads >= kGridEnd)   // n_tiles then is below 2^31, too
    return rkv::fail(RKV_ERR_UNSUPPORTED, "too many sequences for one launch");
  if (int st = check_layout("q", a->q, {a->q_token, a->q_head})) return st;
  return check_layout("out", a->out, {a->out_token, a->out_head});
}

constexpr size_t kRecordBytes = sizeof(int32_t) * 4 * rkv::kAttendShares;

// Rows of a partial sum: those of the largest row tile, made even so that every partial sum (130 floats a row) is 16-byte
// aligned, as its rows are written and read.  groups: a's sequences are groups of sequences, which without cu_q have one row each.
int32_t part_rows(const rkv_pages* p, const rkv_attend* a, bool groups) {
  const int64_t most = (int64_t)(a->cu_q || groups ? a->n_rows : 1) * (a->n_q_heads / p->n_kv_heads);
  return (int32_t)std::min<int64_t>((most + 1) & ~int64_t(1), rkv::kAttendRows);
}

// Rows of the longest sequence, if max_q says so, else of the average one.
int64_t usual_rows(const rkv_pages* p, const rkv_attend* a) {
  return (int64_t)(a->max_q ? a->max_q : (a->n_rows + a->n_seqs - 1) / a->n_seqs) * (a->n_q_heads / p->n_kv_heads);
}

// Whether the row tiles' keys are shared out (attend_shares_kernel and a join) or every tile has a workgroup of its own.
// Shared out, a call pays some 8 us for the list and the join, and rows that are split go through memory; not shared out,
// it lasts as long as its longest tile and leaves CUs idle below 512 tiles.  64 keys take about 0.5 us with at most 16 rows,
// 1 us with more, and at 5.5 TB/s 0.006 us of the whole chip's time.  Measured on 32 query and 8 KV heads, us, not shared
// against shared:
//   one token a sequence: one of 200 keys 9 / 14, of 1024 12 / 15, of 4096 35 / 16, of 32768 250 / 32; 16 of 2048 23 / 33, four
//   of 8192 67 / 33; 64 of 1024 42 / 50, of 2048 92 / 101, of 64 to 8192 127 / 103, of 512 to 8192 187 / 159;
//   prompts: 512 tokens 16 / 34, 1024 27 / 53, 2048 53 / 99, 16384 1997 / 2282; 512 after 32768 568 / 292, 64 after 16320
//   292 / 41, 256 each of four after 7936 200 / 160, 512 each of eight after 3584 258 / 287, 8 each of 16 after 4088 75 / 55.
// Other head layouts go by their items alone.  A call is decided as a whole: one decoding sequence of 131072 keys beside a prompt of 2048
// tokens stays with one workgroup a head (1136 us), and 2304 or 2560 tokens after 32768 take two rounds of tiles (1477, 1502).
bool shared_out(const rkv_pages* p, const rkv_attend* a) {
  const int64_t tiles = row_tiles(p, a), items = tiles * p->n_kv_heads, rows = usual_rows(p, a);
  const int64_t most = (int64_t)a->max_pages * p->page_size;
  if (tiles > rkv::kAttendListed || tiles * std::max<int64_t>(1, (most + 63) / 64) >= kIntEnd || p->n_kv_heads >= (1 << 20))
    return false;   // what the list and its records hold
  const int64_t kv = a->max_kv ? std::min<int64_t>(a->max_kv, most) : most;
  if (rows > rkv::kAttendRows) return items < 512 && kv > 2048;
  if (rows > 16) return kv > (items >= 256 ? 1024 : 512);
  // 3 + 0.5 t us for t tiles of keys against 13 + 0.4 * 0.006 items t where lengths differ as above
  const int64_t t = (kv + 63) / 64;
  return t > 32 || t * (208 - std::min<int64_t>(items, 208)) > 4200;
}

size_t attend_bytes(const rkv_pages* p, const rkv_attend* a) {
  if (nothing_to_do(a) || !shared_out(p, a)) return 0;
  return kRecordBytes + sizeof(float) * 2 * rkv::kAttendShares * (size_t)part_rows(p, a, false) * (rkv::kHeadDim + 2);
}

// 8-bit pools and shared prefixes: whether a launch's key tiles are dealt out (attend_dealt_kernel and a join), by the rule above; of 8-bit pools,
// us, a workgroup per tile against dealt out: one token of one sequence of 1024 12 / 19, of 2048 18.5 / 20, of 4096 31 / 21, of 32768 233 / 32; of 16
// of 2048 21 / 26, of 4096 35 / 40, of 8192 69 / 57; of 64 of 1024 26 and of 2048 45, not dealt out, of 4096 98 / 113, of 3000 to 5000 105 / 112,
// of 512 to 8192 124 / 96, of 64 to 8192 86 / 57.
bool dealt(const rkv_pages* p, const rkv_attend* a) {
  const int64_t tiles = row_tiles(p, a), most = ((int64_t)a->max_pages * p->page_size + 63) / 64;
  if (tiles > rkv::kAttendDealt || tiles * (4 + most) >= kIntEnd || p->n_kv_heads >= (1 << 20)) return false;   // an item's units, and at least one tile
  return shared_out(p, a);
}
// Partial sums of workgroups and of waves: of `rows` rows, the most that a row tile has.
size_t parts_bytes(int32_t rows) {
  return sizeof(float) * (rkv::kHeadDim + 2) * rkv::kAttendShares * (2 * (size_t)rows + 8 * (size_t)std::min(rows, rkv::kAttendFew));
}
// Sums of whole rows, if any, and the records of each row and head, for prefixes and own slots or one of these; rounded up to where partial sums may begin.
size_t rows_bytes(const rkv_attend* a, int sums, int records) {
  return (sizeof(float) * (rkv::kHeadDim * sums + 4 * records) * (size_t)a->n_rows * (size_t)a->n_q_heads + 255) & ~size_t(255);
}
size_t dealt_bytes(const rkv_pages* p, const rkv_attend* a) {
  if (nothing_to_do(a) || !dealt(p, a)) return 0;
  return rows_bytes(a, 0, 1) + parts_bytes(part_rows(p, a, false));
}

// Rows of a call that moves them, and the launch; the rows are written by a read.
int check_rows(const Pool& pool, const rkv_rows* rows, bool written) {
  if (!rows) return rkv::fail(RKV_ERR_INVALID_ARG, "null rows");
  if (rows->n_outer < 0 || rows->n_tokens < 0) return rkv::fail(RKV_ERR_INVALID_ARG, "negative size");
  if (rows->n_outer == 0 || rows->n_tokens == 0) return RKV_OK;
  if (!rows->k || !rows->v || !rows->slots) return rkv::fail(RKV_ERR_INVALID_ARG, "null pointer");
  if ((int64_t)rows->n_outer * rows->n_tokens > 16 * (kGridEnd - 1) / pool.p.n_kv_heads)
    return rkv::fail(RKV_ERR_UNSUPPORTED, "at most 2^28 - 16 rows a call, each head's counted");
  if (int st = check_layout("k rows", rows->k, {rows->k_outer, rows->k_token, rows->k_head})) return st;
  if (int st = check_layout("v rows", rows->v, {rows->v_outer, rows->v_token, rows->v_head})) return st;
  if (written && rows->k == rows->v) return rkv::fail(RKV_ERR_INVALID_ARG, "k and v are read into the same rows");
  const int32_t heads = pool.p.n_kv_heads;
  const Rows k{rows->k, 2, rkv::kHeadDim, {{{rows->k_outer, rows->n_outer}, {rows->k_token, rows->n_tokens}, {rows->k_head, heads}}}};
  const Rows v{rows->v, 2, rkv::kHeadDim, {{{rows->v_outer, rows->n_outer}, {rows->v_token, rows->n_tokens}, {rows->v_head, heads}}}};
  if (written && (!rows_nest(k.dims) || !rows_nest(v.dims)))
    return rkv::fail(RKV_ERR_INVALID_ARG, "the rows to be read into overlap (no stride may be less than the extent of the smaller ones)");
  if (written && rows_meet(k, v))
    return rkv::fail(RKV_ERR_INVALID_ARG, "k's rows to be read into overlap v's (they lie apart, or between each other by the same strides)");
  return RKV_OK;
}
int check_written(const Pool& pool) {
  const rkv_pages& p = pool.p;
  const int size = pool.codes ? 1 : 2;
  auto rows = [&](const void* at, __int128 extent, int64_t page, int64_t head, int64_t slot) {
    return Rows{at, size, extent, {{{page, p.n_pages}, {head, p.n_kv_heads}, {slot, p.page_size}}}};
  };
  const Rows k = rows(p.k, rkv::kHeadDim, p.k_page, p.k_head, p.k_slot), v = rows(p.v, rkv::kHeadDim, p.v_page, p.v_head, p.v_slot);
  const Rows ks = rows(pool.ks.at, 1, pool.ks.page, pool.ks.head, pool.ks.slot), vs = rows(pool.vs.at, 1, pool.vs.page, pool.vs.head, pool.vs.slot);
  bool apart = rows_nest(k.dims) && rows_nest(v.dims);
  if (pool.codes) apart = apart && rows_nest(ks.dims, 1) && rows_nest(vs.dims, 1);
  if (!apart)
    return rkv::fail(RKV_ERR_INVALID_ARG, "the pool's rows overlap (no stride may be less than the extent of the smaller ones): it can be read, not written");
  // A pool whose values are its keys is written twice by the same lanes in order; any other byte that two rows share is a race.
  const bool one = rows_same(k, v) && (!pool.codes || rows_same(ks, vs));
  bool met = !one && rows_meet(k, v);
  if (pool.codes) met = met || (!one && rows_meet(ks, vs)) || rows_meet(k, ks) || rows_meet(k, vs) || rows_meet(v, ks) || rows_meet(v, vs);
  if (met)
    return rkv::fail(RKV_ERR_INVALID_ARG, "k's and v's pages, or their scales, overlap (they lie apart, or between each other by the same strides): they can be read, not written");
  return RKV_OK;
}
rkv::WriteLaunch rows_launch(const Pool& pool, const rkv_rows* rows) {
  rkv::WriteLaunch W{};
  W.p = pool.p;
  W.ks = pool.ks;
  W.vs = pool.vs;
  W.r = *rows;
  W.by_page = rkv::fast_div(pool.p.page_size);
  W.by_head = rkv::fast_div(pool.p.n_kv_heads);
  W.by_token = rkv::fast_div(rows->n_tokens);
  W.n_items = rows->n_outer * rows->n_tokens * pool.p.n_kv_heads;
  W.n_slots = pool.p.n_pages * pool.p.page_size;
  return W;
}
template <class Pages>
int write_rows(const Pages* pages, const rkv_rows* rows, void* stream) {
  rkv::clear_error();
  if (int st = check_pages(pages)) return st;
  const Pool pool = pool_of(pages);
  if (int st = check_rows(pool, rows, false)) return st;
  if (rows->n_outer == 0 || rows->n_tokens == 0) return RKV_OK;
  if (int st = check_written(pool)) return st;
  const rkv::WriteLaunch W = rows_launch(pool, rows);
  return launched(pool.codes ? rkv::launch_write8(W, stream) : rkv::launch_write(W, stream));
}
template <class Pages>
int read_rows(const Pages* pages, const rkv_rows* rows, void* stream) {
  rkv::clear_error();
  if (int st = check_pages(pages)) return st;
  const Pool pool = pool_of(pages);
  if (int st = check_rows(pool, rows, true)) return st;
  if (rows->n_outer == 0 || rows->n_tokens == 0) return RKV_OK;
  const rkv::WriteLaunch W = rows_launch(pool, rows);
  return launched(pool.codes ? rkv::launch_read8(W, stream) : rkv::launch_read(W, stream));
}

// A launch over the row tiles of a call that has been checked, but for its workspace.
rkv::AttendLaunch attend_launch(const Pool& pool, const rkv_attend* a) {
  const rkv_pages* p = &pool.p;
  rkv::AttendLaunch L{};
  L.p = pool.p;
  L.ks = pool.ks;
  L.vs = pool.vs;
  L.a = *a;
  L.group = a->n_q_heads / p->n_kv_heads;
  L.by_page = rkv::fast_div(p->page_size);
  L.by_group = rkv::fast_div(L.group);
  L.n_tiles = (int32_t)row_tiles(p, a);
  L.few_long = 2 * full_tiles(p, a) < L.n_tiles;
  L.n_places = (int32_t)places(p, a);
  L.slot_rows = part_rows(p, a, false);
  // A part of 128 rows is written and read again, as many bytes as four key tiles: not for less than eight.  Few rows
  // cost nothing beside a tile (one token after 1K: 15 us with shares of one, 17 of four, 21 of eight).
  L.least = usual_rows(p, a) > 32 ? 8 : 1;
  return L;
}
void set_parts(rkv::AttendLaunch& L, int32_t rows, char* at) {
  L.slot_rows = rows;
  L.few_rows = std::min(rows, rkv::kAttendFew);
  L.parts = reinterpret_cast<float*>(at);
  L.few_parts = L.parts + 2 * (size_t)rkv::kAttendShares * rows * (rkv::kHeadDim + 2);
}
int check_workspace(size_t need, const void* ws, size_t ws_bytes) {
  if (need && !ws) return rkv::fail(RKV_ERR_WORKSPACE, "workspace is null");
  if (need && (uintptr_t)ws % 256) return rkv::fail(RKV_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  if (ws_bytes < need) return rkv::fail(RKV_ERR_WORKSPACE, "workspace too small: need " + std::to_string(need) + " bytes");
  return RKV_OK;
}

// A launch without prefixes, in a workspace of what it needs.
int launch_alone(const Pool& pool, const rkv_attend* a, size_t need, char* ws, void* stream) {
  rkv::AttendLaunch L = attend_launch(pool, a);
  if (pool.codes) {
    if (need) {
      L.sum_records = reinterpret_cast<float*>(ws);
      set_parts(L, part_rows(&pool.p, a, false), ws + rows_bytes(a, 0, 1));
    }
    return rkv::launch_attend8(L, stream);
  }
  if (need) {
    L.records = reinterpret_cast<int32_t*>(ws);
    L.parts = reinterpret_cast<float*>(ws + kRecordBytes);
  }
  return rkv::launch_attend(L, stream);
}

template <class Pages>
int attend_size(const Pages* pages, const rkv_attend* a, size_t* bytes) {
  rkv::clear_error();
  if (!bytes) return rkv::fail(RKV_ERR_INVALID_ARG, "null pointer");
  if (int st = check_pages(pages)) return st;
  const Pool pool = pool_of(pages);
  if (int st = check_attend(&pool.p, a, pool.codes ? dealt : shared_out)) return st;
  *bytes = pool.codes ? dealt_bytes(&pool.p, a) : attend_bytes(&pool.p, a);
  return RKV_OK;
}
template <class Pages>
int attend(const Pages* pages, const rkv_attend* a, void* ws, size_t ws_bytes, void* stream) {
  rkv::clear_error();
  if (int st = check_pages(pages)) return st;
  const Pool pool = pool_of(pages);
  if (int st = check_attend(&pool.p, a, pool.codes ? dealt : shared_out)) return st;
  if (nothing_to_do(a)) return RKV_OK;
  if (!a->q || !a->out || !a->lens || (a->max_pages && !a->table)) return rkv::fail(RKV_ERR_INVALID_ARG, "null pointer");
  const size_t need = pool.codes ? dealt_bytes(&pool.p, a) : attend_bytes(&pool.p, a);
  if (int st = check_workspace(need, ws, ws_bytes)) return st;
  return launched(launch_alone(pool, a, need, static_cast<char*>(ws), stream));
}

// ---- shared prefixes: the groups' rows over their prefixes, then each sequence's rows over its own slots, from those sums on

// The call over the prefixes.  A group's rows are those of all its sequences.
rkv_attend over_prefixes(const rkv_attend* a, const rkv_shared* g) {
  rkv_attend b = *a;
  b.table = g->table;
  b.table_stride = g->table_stride;
  b.lens = g->lens;
  b.prefix_lens = b.first_keys = nullptr;
  b.n_seqs = g->n_groups;
  b.max_pages = g->max_pages;
  b.max_q = 0;     // the groups' rows on average
  b.max_kv = g->max_len;
  return b;
}
int check_shared(const rkv_pages* p, const rkv_attend* a, const rkv_shared* g) {
  if (int st = check_attend(p, a, dealt)) return st;
  if (!g) return rkv::fail(RKV_ERR_INVALID_ARG, "null shared");
  if (g->n_groups < 0 || g->max_pages < 0 || g->max_len < 0 || g->table_stride < 0) return rkv::fail(RKV_ERR_INVALID_ARG, "negative size");
  if (a->prefix_lens || a->first_keys) return rkv::fail(RKV_ERR_UNSUPPORTED, "prefix_lens and first_keys do not go with shared prefixes");
  if (g->table_stride < g->max_pages) return rkv::fail(RKV_ERR_SHAPE, "the shared table's stride is less than its max_pages");
  if (((int64_t)g->max_pages + a->max_pages) * p->page_size >= kIntEnd - 1024)
    return rkv::fail(RKV_ERR_UNSUPPORTED, "a prefix and a sequence hold fewer than 2^31 - 1024 slots together");
  const rkv_attend b = over_prefixes(a, g);
  if (!nothing_to_do(&b) && !dealt(p, &b) && places(p, &b) * p->n_kv_heads >= kGridEnd)
    return rkv::fail(RKV_ERR_UNSUPPORTED, "too many groups for one launch");
  return RKV_OK;
}
// Whether one launch takes both: the rows of all sequences over the prefixes and those of each over its own slots in one list, all sums by way
// of memory and one join.  Two launches, one after the other, pay for two lists and two ramps, but only the prefixes' sums go through
// memory and full rows are finished where they are.  Measured on 32 query and 8 KV heads, sequences x tokens behind a prefix, 64 to 512 own slots, us,
// one against two: 16 x 1 behind 1024 24 / 36, 64 x 1 behind 8192 42 / 56, 64 x 8 115 / 118, 8 x 64 111 / 112, 64 x 16 194 / 187, 64 x 32 369 / 302;
// 16 x 32 behind 1024 44 / 48, 16 x 64 61 / 53; in 8 bits 64 x 1 44 / 59, 64 x 8 122 / 125, 8 x 64 116 / 118, 64 x 16 200 / 197, 64 x 32 376 / 320;
// 16 x 32 behind 1024 46 / 49, 16 x 64 64 / 56.
bool both_at_once(const rkv_pages* p, const rkv_attend* a, const rkv_attend* b) {
  const int64_t own = row_tiles(p, a), over = row_tiles(p, b), rows = (int64_t)a->n_rows * (a->n_q_heads / p->n_kv_heads);
  auto tiles = [&](int64_t pages) { return 4 + (pages * p->page_size + 63) / 64; };
  return rows <= 2048 && own + over <= rkv::kAttendDealt && own * tiles(a->max_pages) + over * tiles(b->max_pages) < kIntEnd &&
         p->n_kv_heads < (1 << 20);
}
size_t shared_bytes(const rkv_pages* p, const rkv_attend* a, const rkv_shared* g, bool codes) {
  const rkv_attend b = over_prefixes(a, g);
  if (nothing_to_do(a) || nothing_to_do(&b)) return codes ? dealt_bytes(p, a) : attend_bytes(p, a);
  if (both_at_once(p, a, &b)) return rows_bytes(a, 2, 2) + parts_bytes(part_rows(p, &b, true));
  return rows_bytes(a, 1, 1) + std::max(dealt(p, a) ? parts_bytes(part_rows(p, a, false)) : 0, dealt(p, &b) ? parts_bytes(part_rows(p, &b, true)) : 0);
}

template <class Pages>
int shared_size(const Pages* pages, const rkv_attend* a, const rkv_shared* g, size_t* bytes) {
  rkv::clear_error();
  if (!bytes) return rkv::fail(RKV_ERR_INVALID_ARG, "null pointer");
  if (int st = check_pages(pages)) return st;
  const Pool pool = pool_of(pages);
  if (int st = check_shared(&pool.p, a, g)) return st;
  *bytes = shared_bytes(&pool.p, a, g, pool.codes);
  return RKV_OK;
}
template <class Pages>
int attend_shared(const Pages* pages, const rkv_attend* a, const rkv_shared* g, void* ws, size_t ws_bytes, void* stream) {
  rkv::clear_error();
  if (int st = check_pages(pages)) return st;
  const Pool pool = pool_of(pages);
  const rkv_pages* p = &pool.p;
  if (int st = check_shared(p, a, g)) return st;
  if (nothing_to_do(a)) return RKV_OK;
  if (!a->q || !a->out || !a->lens || (a->max_pages && !a->table) || (g->n_groups && (!g->lens || !g->cu_seqs || (g->max_pages && !g->table))))
    return rkv::fail(RKV_ERR_INVALID_ARG, "null pointer");
  const size_t need = shared_bytes(p, a, g, pool.codes);
  if (int st = check_workspace(need, ws, ws_bytes)) return st;
  const rkv_attend b = over_prefixes(a, g);
  if (nothing_to_do(&b)) return launched(launch_alone(pool, a, need, static_cast<char*>(ws), stream));
  auto* launch = pool.codes ? rkv::launch_attend8_shared : rkv::launch_attend_shared;
  const bool both = both_at_once(p, a, &b);
  rkv::AttendLaunch L = attend_launch(pool, a);
  L.g = *g;
  L.sums = static_cast<float*>(ws);
  L.sum_records = L.sums + (both ? 2 : 1) * (size_t)a->n_rows * a->n_q_heads * rkv::kHeadDim;
  char* rest = static_cast<char*>(ws) + rows_bytes(a, both ? 2 : 1, both ? 2 : 1);
  if (both) {
    L.stage = rkv::kBoth;
    L.n_group_tiles = (int32_t)row_tiles(p, &b);
    L.n_tiles += L.n_group_tiles;
    L.least = 1;
    set_parts(L, part_rows(p, &b, true), rest);
    return launched(launch(L, stream));
  }
  const rkv::AttendLaunch tiles = attend_launch(pool, &b);
  rkv::AttendLaunch G = L;
  G.n_tiles = G.n_group_tiles = tiles.n_tiles;
  G.few_long = tiles.few_long;
  G.n_places = tiles.n_places;
  G.least = tiles.least;
  G.stage = rkv::kOverPrefix;
  L.stage = rkv::kOverOwn;
  if (dealt(p, &b)) set_parts(G, part_rows(p, &b, true), rest);
  if (dealt(p, a)) set_parts(L, part_rows(p, a, false), rest);
  if (int st = launched(launch(G, stream))) return st;
  return launched(launch(L, stream));
}

}  // namespace

extern "C" {

int rkv_pages_resize(const rkv_resize* r, void* stream) {
  rkv::clear_error();
  if (!r) return rkv::fail(RKV_ERR_INVALID_ARG, "null resize");
  if (r->n_seqs < 0 || r->max_pages < 0 || r->max_new < 0 || r->table_stride < 0 || r->n_pages < 1 || r->page_size < 1)
    return rkv::fail(RKV_ERR_INVALID_ARG, "negative size, or no pages");
  if (!r->ring || !r->cursor || !r->cursor_out || !r->cu_new || !r->status || (r->max_new && !r->slots) ||
      (r->n_seqs && (!r->lens || !r->new_lens || !r->lens_out)) || (r->n_seqs && r->max_pages && !r->table))
    return rkv::fail(RKV_ERR_INVALID_ARG, "null pointer");
  if (r->n_seqs > rkv::kResizeMaxSeqs)
    return rkv::fail(RKV_ERR_UNSUPPORTED, "at most " + std::to_string(rkv::kResizeMaxSeqs) + " sequences");
  if ((int64_t)r->n_pages * r->page_size >= kIntEnd || (int64_t)r->max_pages * r->page_size >= kIntEnd)
    return rkv::fail(RKV_ERR_UNSUPPORTED, "a pool and a sequence hold fewer than 2^31 slots");
  if (r->table_stride < r->max_pages) return rkv::fail(RKV_ERR_SHAPE, "table_stride is less than max_pages");
  return launched(rkv::launch_resize({*r, rkv::fast_div(r->page_size)}, stream));
}

int rkv_pages_write(const rkv_pages* pages, const rkv_rows* rows, void* stream) { return write_rows(pages, rows, stream); }
int rkv_qpages_write(const rkv_qpages* pages, const rkv_rows* rows, void* stream) { return write_rows(pages, rows, stream); }

int rkv_pages_read(const rkv_pages* pages, const rkv_rows* rows, void* stream) { return read_rows(pages, rows, stream); }
int rkv_qpages_read(const rkv_qpages* pages, const rkv_rows* rows, void* stream) { return read_rows(pages, rows, stream); }

int rkv_pages_attend_workspace_size(const rkv_pages* pages, const rkv_attend* a, size_t* bytes) { return attend_size(pages, a, bytes); }
int rkv_qpages_attend_workspace_size(const rkv_qpages* pages, const rkv_attend* a, size_t* bytes) { return attend_size(pages, a, bytes); }

int rkv_pages_attend(const rkv_pages* pages, const rkv_attend* a, void* ws, size_t ws_bytes, void* stream) {
  return attend(pages, a, ws, ws_bytes, stream);
}
int rkv_qpages_attend(const rkv_qpages* pages, const rkv_attend* a, void* ws, size_t ws_bytes, void* stream) {
  return attend(pages, a, ws, ws_bytes, stream);
}

int rkv_pages_attend_shared_workspace_size(const rkv_pages* pages, const rkv_attend* a, const rkv_shared* shared, size_t* bytes) {
  return shared_size(pages, a, shared, bytes);
}
int rkv_qpages_attend_shared_workspace_size(const rkv_qpages* pages, const rkv_attend* a, const rkv_shared* shared, size_t* bytes) {
  return shared_size(pages, a, shared, bytes);
}
int rkv_pages_attend_shared(const rkv_pages* pages, const rkv_attend* a, const rkv_shared* shared, void* ws, size_t ws_bytes, void* stream) {
  return attend_shared(pages, a, shared, ws, ws_bytes, stream);
}
int rkv_qpages_attend_shared(const rkv_qpages* pages, const rkv_attend* a, const rkv_shared* shared, void* ws, size_t ws_bytes, void* stream) {
  return attend_shared(pages, a, shared, ws, ws_bytes, stream);
}

}  // extern "C"
