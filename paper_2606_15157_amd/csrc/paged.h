// Declarations of the paged caches: paged.cpp checks, pages.hip moves rows and the attend*.hip instances of attend_rows.h and attend_dealt.h compute.
#pragma once

#include "rkv_internal.h"

namespace rkv {

// n / d for 0 <= n < 2^31 and 1 <= d < 2^31: with l = ceil(log2 d) and mul = ceil(2^(31 + l) / d), the product
// n mul exceeds n 2^(31 + l) / d by n (d mul - 2^(31 + l)) / d < n 2^l / d, less than 2^(31 + l) / d: the floor is exact.
struct FastDiv {
  uint32_t mul, shift;
};
inline FastDiv fast_div(int32_t d) {
  uint32_t l = 0;
  while ((1ull << l) < (uint64_t)d) ++l;
  return {(uint32_t)(((1ull << (31 + l)) + (uint64_t)d - 1) / (uint64_t)d), l};
}

constexpr int kResizeMaxSeqs = 8192;       // sequences whose three prefix sums one workgroup keeps in LDS
struct ResizeLaunch {
  rkv_resize r;
  FastDiv by_page;
};
int launch_resize(const ResizeLaunch& R, void* stream);

struct Scales {      // exponent bytes of an 8-bit pool's rows
  uint8_t* at;
  int64_t page, head, slot;
};

// Rows to slots, and back.
struct WriteLaunch {
  rkv_pages p;         // an 8-bit pool's strides are of its codes
  Scales ks, vs;
  rkv_rows r;          // a read writes them
  FastDiv by_page, by_head, by_token;
  int32_t n_items;     // n_outer * n_tokens * n_kv_heads
  int32_t n_slots;
};
int launch_write(const WriteLaunch& W, void* stream);
int launch_write8(const WriteLaunch& W, void* stream);
int launch_read(const WriteLaunch& W, void* stream);
int launch_read8(const WriteLaunch& W, void* stream);

constexpr int kAttendRows = 128;       // rows (tokens x query heads of a group) of a tile
constexpr int kAttendShares = 512;     // workgroups that share the key tiles of a short list of row tiles: two a CU
constexpr int kAttendListed = 1024;    // row tiles such a list may have
constexpr int kAttendDealt = 768;      // and one of 8-bit pools or shared prefixes
constexpr int kAttendFew = 16;         // rows that a wave takes by itself there
// The launches of a call whose sequences share prefixes: over the prefixes, and over the own slots from the sums of the first on; or over both, whose
// sums a join brings together.
enum { kAlone = 0, kOverPrefix = 1, kOverOwn = 2, kBoth = 3 };
struct AttendLaunch {
  rkv_pages p;         // an 8-bit pool's strides are of its codes
  Scales ks, vs;
  rkv_attend a;
  FastDiv by_page, by_group;
  int32_t group;       // Hq / Hkv
  int32_t n_tiles;     // row tiles of all sequences, at most
  int32_t n_places;    // places of attend_tiles_kernel: n_seqs, then numbers of long sequences' tiles
  int32_t few_long;    // how those are numbered
  int32_t slot_rows;   // rows of a partial sum, an even number
  int32_t least;       // key tiles of a share, at least
  int32_t* records;    // [kAttendShares][4], then
  float* parts;        // [2 kAttendShares] partial sums; null: a workgroup per row tile
  int32_t few_rows;    // of a wave's partial sum, an even number
  float* few_parts;    // [8 kAttendShares] of these
  // Shared prefixes.  Row tiles of the groups are those of all their sequences' rows; a launch has the tiles of the groups, of the
  // sequences, or of both (the groups' first).
  int32_t stage;
  int32_t n_group_tiles;      // of n_tiles
  rkv_shared g;
  float* sums;                // [n_rows][Hq][128] over the prefixes, with kBoth then over the own slots
  float* sum_records;         // [n_rows][Hq][4], likewise
};
// 16-bit and 8-bit pools, without and with shared prefixes.
int launch_attend(const AttendLaunch& A, void* stream);
int launch_attend8(const AttendLaunch& A, void* stream);
int launch_attend_shared(const AttendLaunch& A, void* stream);
int launch_attend8_shared(const AttendLaunch& A, void* stream);

}  // namespace rkv
