// Parameters of the page bookkeeping kernels.
#pragma once

#include "hswa_internal.cuh"

// Limits of one call: rows of a table and pages of a pool whose bookkeeping fits a cluster's shared memory, and entries of a table
// whose number of fresh pages fits 32 bits.
constexpr int kMaxPageRows = 4096, kMaxPages = 1 << 23;
constexpr int64_t kMaxPageEntries = 1 << 30;
constexpr int kPoolsPerLaunch = 64;

struct PagesForkParams {
  int32_t num_pages, page_size;
  const int32_t* ref;  // [num_pages] holders of each page
  int32_t* ref_out;
  int32_t rows_in;
  const int32_t* held;   // [rows_in] pages of each row
  const int32_t* table;  // [rows_in][max_blocks]
  int32_t max_blocks;
  int32_t rows_out;
  const int32_t* parent;  // [rows_out]
  const int32_t* len;
  const int32_t* need;
  int32_t* table_out;  // [rows_out][out_max_blocks]
  int32_t out_max_blocks;
  int32_t* held_out;  // [rows_out]
  int32_t* copy_src;
  int32_t* copy_dst;
  // scratch: the fresh pages [num_pages]; for a second launch [kMaxPageRows] each: first child and most pages a child shares of
  // each old row, rank of each new row's first fresh page; whether there is anything to do
  int32_t *fresh, *first, *most, *rank, *ok;
  int32_t second;
  int32_t copied;  // the counts are copied, and the bitmap of free pages put into `fresh`, by a launch before
  int32_t* err;
};

struct PagesCompactParams {
  int32_t num_pages;
  const int32_t* ref;
  int32_t* ref_out;
  int32_t rows;
  const int32_t* held;
  const int32_t* table;
  int32_t max_blocks;
  int32_t* table_out;
  int32_t* page_map;  // [num_pages]
  int32_t max_moves;
  int32_t* move_src;
  int32_t* move_dst;
  int32_t second;  // the tables are rewritten by a second launch
  int32_t copied;  // the counts are copied, the map set to the identity, and the bitmap put into its first entries, by a launch before
  int32_t* err;
};

struct PagesCopyParams {
  void* pools[kPoolsPerLaunch];
  int32_t n_pools;
  int64_t page_bytes;
  int64_t num_pages;
  int32_t pairs;
  const int32_t* src;
  const int32_t* dst;
  int32_t* err;
};

cudaError_t hswa_launch_pages_fork(const PagesForkParams& p, int num_sms, cudaStream_t s);
cudaError_t hswa_launch_pages_compact(const PagesCompactParams& p, int num_sms, cudaStream_t s);
cudaError_t hswa_launch_pages_copy(const PagesCopyParams& p, cudaStream_t s);
