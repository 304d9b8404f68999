// Host side of the paged caches: argument checks and launches of rkv_pages_resize, rkv_pages_write and
// rkv_pages_attend.
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

// A 16-byte aligned pointer and strides (elements) of whole 16-byte pieces.
int check_layout(const char* what, const void* ptr, std::initializer_list<int64_t> strides) {
  for (int64_t s : strides)
    if (s < 0) return rkv::fail(RKV_ERR_INVALID_ARG, std::string(what) + ": negative stride");
  if ((uintptr_t)ptr % 16) return rkv::fail(RKV_ERR_UNSUPPORTED, std::string(what) + " must be 16-byte aligned");
  for (int64_t s : strides)
    if (s % 8) return rkv::fail(RKV_ERR_UNSUPPORTED, std::string(what) + ": strides must be multiples of 8 elements");
  return RKV_OK;
}

// Whether rows of 128 elements, at sum_i index_i stride_i for index_i < count_i, are told apart by their dimensions: taken by
// stride, each is at least the extent of the smaller ones.  So are those of every slice and permutation of a dense tensor.
struct Dim {
  int64_t stride, count;
};
template <size_t kDims>
bool rows_nest(std::array<Dim, kDims> dims) {
  std::sort(dims.begin(), dims.end(), [](const Dim& x, const Dim& y) { return x.stride < y.stride; });
  __int128 extent = rkv::kHeadDim;
  for (const Dim& d : dims) {
    if (d.count <= 1) continue;
    if (d.stride < extent) return false;
    extent += (__int128)d.stride * (d.count - 1);
  }
  return true;
}

int check_pages(const rkv_pages* p) {
  if (!p) return rkv::fail(RKV_ERR_INVALID_ARG, "null pages");
  if (!p->k || !p->v) return rkv::fail(RKV_ERR_INVALID_ARG, "null page pool");
  if (p->n_pages < 1 || p->page_size < 1 || p->n_kv_heads < 1)
    return rkv::fail(RKV_ERR_INVALID_ARG, "n_pages, page_size and n_kv_heads must be >= 1");
  if (p->dtype != RKV_BF16 && p->dtype != RKV_F16) return rkv::fail(RKV_ERR_INVALID_ARG, "unknown dtype");
  if (p->head_dim != rkv::kHeadDim) return rkv::fail(RKV_ERR_UNSUPPORTED, "head_dim must be 128");
  if ((int64_t)p->n_pages * p->page_size >= kIntEnd) return rkv::fail(RKV_ERR_UNSUPPORTED, "a pool holds fewer than 2^31 slots");
  if (p->k_slot >= kIntEnd / 16 || p->v_slot >= kIntEnd / 16)
    return rkv::fail(RKV_ERR_UNSUPPORTED, "slots are fewer than 2^27 elements apart");
  if (int st = check_layout("k pages", p->k, {p->k_page, p->k_head, p->k_slot})) return st;
  return check_layout("v pages", p->v, {p->v_page, p->v_head, p->v_slot});
}

// Row tiles, with one part-filled tile for each sequence.
int64_t full_tiles(const rkv_pages* p, const rkv_attend* a) { return (int64_t)a->n_rows * (a->n_q_heads / p->n_kv_heads) / rkv::kAttendRows; }
int64_t row_tiles(const rkv_pages* p, const rkv_attend* a) { return full_tiles(p, a) + a->n_seqs; }

// Places of attend_tiles_kernel: the sequences, then the numbers of long sequences' tiles.
int64_t places(const rkv_pages* p, const rkv_attend* a) { return a->n_seqs + std::min(2 * full_tiles(p, a), row_tiles(p, a)); }
bool nothing_to_do(const rkv_attend* a) { return a->n_seqs == 0 || a->n_rows == 0; }
bool shared_out(const rkv_pages* p, const rkv_attend* a);

int check_attend(const rkv_pages* p, const rkv_attend* a) {
  if (int st = check_pages(p)) return st;
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
  if (!nothing_to_do(a) && !shared_out(p, a) && places(p, a) * p->n_kv_heads >= kGridEnd)   // n_tiles then is below 2^31, too
    return rkv::fail(RKV_ERR_UNSUPPORTED, "too many sequences for one launch");
  if (int st = check_layout("q", a->q, {a->q_token, a->q_head})) return st;
  return check_layout("out", a->out, {a->out_token, a->out_head});
}

constexpr size_t kRecordBytes = sizeof(int32_t) * 4 * rkv::kAttendShares;

// Rows of a partial sum: those of the largest row tile, made even so that every partial sum (130 floats a row) is 16-byte
// aligned, as its rows are written and read.
int32_t part_rows(const rkv_pages* p, const rkv_attend* a) {
  const int64_t most = (int64_t)(a->cu_q ? a->n_rows : 1) * (a->n_q_heads / p->n_kv_heads);
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
  return kRecordBytes + sizeof(float) * 2 * rkv::kAttendShares * (size_t)part_rows(p, a) * (rkv::kHeadDim + 2);
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

int rkv_pages_write(const rkv_pages* pages, const rkv_rows* rows, void* stream) {
  rkv::clear_error();
  if (int st = check_pages(pages)) return st;
  if (!rows) return rkv::fail(RKV_ERR_INVALID_ARG, "null rows");
  if (rows->n_outer < 0 || rows->n_tokens < 0) return rkv::fail(RKV_ERR_INVALID_ARG, "negative size");
  if (rows->n_outer == 0 || rows->n_tokens == 0) return RKV_OK;
  if (!rows->k || !rows->v || !rows->slots) return rkv::fail(RKV_ERR_INVALID_ARG, "null pointer");
  if ((int64_t)rows->n_outer * rows->n_tokens > 16 * (kGridEnd - 1) / pages->n_kv_heads)
    return rkv::fail(RKV_ERR_UNSUPPORTED, "at most 2^28 - 16 rows a call, each head's counted");
  if (int st = check_layout("k rows", rows->k, {rows->k_outer, rows->k_token, rows->k_head})) return st;
  if (int st = check_layout("v rows", rows->v, {rows->v_outer, rows->v_token, rows->v_head})) return st;
  const rkv_pages& p = *pages;
  if (!rows_nest<3>({{{p.k_page, p.n_pages}, {p.k_head, p.n_kv_heads}, {p.k_slot, p.page_size}}}) ||
      !rows_nest<3>({{{p.v_page, p.n_pages}, {p.v_head, p.n_kv_heads}, {p.v_slot, p.page_size}}}))
    return rkv::fail(RKV_ERR_INVALID_ARG, "the pool's rows overlap (no stride may be less than the extent of the smaller ones): it can be read, not written");
  rkv::WriteLaunch W{};
  W.p = *pages;
  W.r = *rows;
  W.by_page = rkv::fast_div(pages->page_size);
  W.by_head = rkv::fast_div(pages->n_kv_heads);
  W.by_token = rkv::fast_div(rows->n_tokens);
  W.n_items = rows->n_outer * rows->n_tokens * pages->n_kv_heads;
  W.n_slots = pages->n_pages * pages->page_size;
  return launched(rkv::launch_write(W, stream));
}

int rkv_pages_attend_workspace_size(const rkv_pages* pages, const rkv_attend* a, size_t* bytes) {
  rkv::clear_error();
  if (!bytes) return rkv::fail(RKV_ERR_INVALID_ARG, "null pointer");
  if (int st = check_attend(pages, a)) return st;
  *bytes = attend_bytes(pages, a);
  return RKV_OK;
}

int rkv_pages_attend(const rkv_pages* pages, const rkv_attend* a, void* ws, size_t ws_bytes, void* stream) {
  rkv::clear_error();
  if (int st = check_attend(pages, a)) return st;
  if (nothing_to_do(a)) return RKV_OK;
  if (!a->q || !a->out || !a->lens || (a->max_pages && !a->table)) return rkv::fail(RKV_ERR_INVALID_ARG, "null pointer");
  const size_t need = attend_bytes(pages, a);
  if (need && !ws) return rkv::fail(RKV_ERR_WORKSPACE, "workspace is null");
  if (need && (uintptr_t)ws % 256) return rkv::fail(RKV_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  if (ws_bytes < need) return rkv::fail(RKV_ERR_WORKSPACE, "workspace too small: need " + std::to_string(need) + " bytes");
  rkv::AttendLaunch L{};
  L.p = *pages;
  L.a = *a;
  L.group = a->n_q_heads / pages->n_kv_heads;
  L.by_page = rkv::fast_div(pages->page_size);
  L.by_group = rkv::fast_div(L.group);
  L.n_tiles = (int32_t)row_tiles(pages, a);
  L.few_long = 2 * full_tiles(pages, a) < L.n_tiles;
  L.n_places = (int32_t)places(pages, a);
  L.slot_rows = part_rows(pages, a);
  // A part of 128 rows is written and read again, as many bytes as four key tiles: not for less than eight.  Few rows
  // cost nothing beside a tile (one token after 1K: 15 us with shares of one, 17 of four, 21 of eight).
  L.least = usual_rows(pages, a) > 32 ? 8 : 1;
  if (need) {
    L.records = static_cast<int32_t*>(ws);
    L.parts = reinterpret_cast<float*>(static_cast<char*>(ws) + kRecordBytes);
  }
  return launched(rkv::launch_attend(L, stream));
}

}  // extern "C"
