// Declarations of the paged caches: paged.cpp checks, pages.hip and attend.hip compute.
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

struct WriteLaunch {
  rkv_pages p;
  rkv_rows r;
  FastDiv by_page, by_head, by_token;
  int32_t n_items;     // n_outer * n_tokens * n_kv_heads
  int32_t n_slots;
};
int launch_write(const WriteLaunch& W, void* stream);

constexpr int kAttendRows = 128;       // rows (tokens x query heads of a group) of a tile
constexpr int kAttendShares = 512;     // workgroups that share the key tiles of a short list of row tiles: two a CU
constexpr int kAttendListed = 1024;    // row tiles such a list may have
struct AttendLaunch {
  rkv_pages p;
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
};
int launch_attend(const AttendLaunch& A, void* stream);

}  // namespace rkv
