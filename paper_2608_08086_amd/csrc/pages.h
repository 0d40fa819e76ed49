// Pages of a paged cache that several sequences share: kernel arguments and launchers.
//
// refs[p] counts the table rows that hold page p; a page without a holder is in the ring of
// free pages or, while a call is at work, on its way there.
#pragma once

#include "common.h"

constexpr int PAGES_MAX_ROWS = 4096;        // requests of a plan, forks of a call
constexpr int PAGES_MAX_TABLE = 65536;      // table rows of a fork (a bit each in LDS)
constexpr int PAGES_BLOCK = 2048;           // pages of a workgroup of the compaction

struct PagesForkArgs {
  int n;
  const int *src, *dst, *len;
  int psh, n_pages, n_rows, width;
  int* table;
  const int* refs_in;
  int *refs_out, *status;
};

struct PagesPlanArgs {
  int batch;
  const int *len_old, *len_new;
  int psh, n_pages, width;
  const int* table_in;
  int *table_out, *free_pages;
  const int* pool_in;
  int* pool_out;
  const int* refs_in;
  int *refs_out, *row_off, *slots;
  int slot_rows;
  int *copy_src, *copy_dst, *status;
  // workspace: what the call does to a page (drops, writers << 16), the last row that does,
  // per row the pages it gives back and whether it copies, and whether an entry is bad
  int *todo, *last, *given, *copies, *bad;
};

struct PagesCompactArgs {
  int batch;
  const int* len;
  int psh, n_pages, width;
  const int* table_in;
  int* table_out;
  const int* refs_in;
  int *refs_out, *free_pages, *pool_out, *move_src, *move_dst, *moves;
  int *used, *rank;      // workspace: pages in use of each block, a moved page's place among the moves
};

struct PagesCopyArgs {
  char* data;
  long page_bytes, plane_stride;
  int n_pages, planes, n;
  const int *src, *dst, *count;
};

void launch_pages_fork(const PagesForkArgs& a, hipStream_t st);
void launch_pages_plan(const PagesPlanArgs& a, hipStream_t st);
void launch_pages_compact(const PagesCompactArgs& a, hipStream_t st);
void launch_pages_copy(const PagesCopyArgs& a, hipStream_t st);
