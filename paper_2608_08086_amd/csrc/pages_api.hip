// Entry points of the pages that several sequences share (archer_ops.h):
// host-side checks, then the launches.
#include "archer_ops.h"
#include "errors.h"
#include "host_checks.h"
#include "pages.h"

namespace {

#define HIPCHK(x)                                                                                              \
  do {                                                                                                         \
    hipError_t e_ = (x);                                                                                       \
    if (e_ != hipSuccess) return archer_fail(ARCHER_E_HIP, std::string(#x) + ": " + hipGetErrorString(e_));    \
  } while (0)

const char* table_error(int32_t max_pages, int32_t page_size) {
  if (max_pages < 1 || (long long)max_pages * page_size > INT_MAX) return "max_pages must be positive, max_pages * page_size below 2^31";
  return nullptr;
}

// an output that may be its input, but not overlap it otherwise
bool overlaps(const int32_t* in, const int32_t* out, long long n) { return in != out && in < out + n && out < in + n; }

archer_status check_workspace(const void* ws, size_t have, size_t need) {
  if (!ws || ((uintptr_t)ws & 255) || have < need) return archer_fail(ARCHER_E_WORKSPACE, "workspace too small or misaligned");
  return ARCHER_OK;
}

}  // namespace

extern "C" {

archer_status archer_pages_fork(int32_t n, const int32_t* src, const int32_t* dst, const int32_t* len, int32_t page_size,
                                int32_t n_pages, int32_t n_rows, int32_t max_pages, int32_t* table, const int32_t* refs_in,
                                int32_t* refs_out, int32_t* status, void* hip_stream) {
  if (!src || !dst || !len || !table || !refs_in || !refs_out || !status) return archer_fail(ARCHER_E_ARG, "null argument");
  if (n < 1 || n > PAGES_MAX_ROWS) return archer_fail(ARCHER_E_SHAPE, "n must be in [1, 4096]");
  if (n_rows < 1 || n_rows > PAGES_MAX_TABLE) return archer_fail(ARCHER_E_SHAPE, "n_rows must be in [1, 65536]");
  if (const char* e = pages_error(page_size, n_pages)) return archer_fail(ARCHER_E_SHAPE, e);
  if (const char* e = table_error(max_pages, page_size)) return archer_fail(ARCHER_E_SHAPE, e);
  if (overlaps(refs_in, refs_out, n_pages)) return archer_fail(ARCHER_E_ARG, "refs_out must be refs_in or not overlap it");
  PagesForkArgs a;
  a.n = n; a.src = src; a.dst = dst; a.len = len;
  a.psh = page_shift(page_size); a.n_pages = n_pages; a.n_rows = n_rows; a.width = max_pages;
  a.table = table; a.refs_in = refs_in; a.refs_out = refs_out; a.status = status;
  launch_pages_fork(a, (hipStream_t)hip_stream);
  HIPCHK(hipGetLastError());
  return ARCHER_OK;
}

size_t archer_pages_plan_ws_bytes(int32_t batch, int32_t n_pages) {
  if (batch < 1 || batch > PAGES_MAX_ROWS || n_pages < 1) return 0;
  return align_up(((size_t)n_pages * 2 + (size_t)batch * 2 + 1) * 4, 256);
}

archer_status archer_pages_plan(int32_t batch, const int32_t* len_old, const int32_t* len_new, int32_t page_size,
                                int32_t n_pages, int32_t max_pages, const int32_t* table_in, int32_t* table_out,
                                int32_t* free_pages, const int32_t* pool_in, int32_t* pool_out, const int32_t* refs_in,
                                int32_t* refs_out, int32_t* row_off, int32_t* slot_map, int32_t slot_rows,
                                int32_t* copy_src, int32_t* copy_dst, int32_t* status, void* workspace, size_t ws_bytes,
                                void* hip_stream) {
  if (!len_old || !len_new || !table_in || !table_out || !free_pages || !pool_in || !pool_out || !refs_in || !refs_out ||
      !row_off || !copy_src || !copy_dst || !status || (!slot_map && slot_rows > 0))
    return archer_fail(ARCHER_E_ARG, "null argument");
  if (batch < 1 || batch > PAGES_MAX_ROWS) return archer_fail(ARCHER_E_SHAPE, "batch must be in [1, 4096]");
  if (const char* e = pages_error(page_size, n_pages)) return archer_fail(ARCHER_E_SHAPE, e);
  if (const char* e = table_error(max_pages, page_size)) return archer_fail(ARCHER_E_SHAPE, e);
  if (slot_rows < 0) return archer_fail(ARCHER_E_SHAPE, "slot_rows must not be negative");
  if (pool_in < pool_out + 2 && pool_out < pool_in + 2) return archer_fail(ARCHER_E_ARG, "pool_out must not alias pool_in");
  if (overlaps(table_in, table_out, (long long)batch * max_pages) || overlaps(refs_in, refs_out, n_pages))
    return archer_fail(ARCHER_E_ARG, "table_out and refs_out must be table_in and refs_in or not overlap them");
  if (archer_status s = check_workspace(workspace, ws_bytes, archer_pages_plan_ws_bytes(batch, n_pages))) return s;
  PagesPlanArgs a;
  a.batch = batch; a.len_old = len_old; a.len_new = len_new;
  a.psh = page_shift(page_size); a.n_pages = n_pages; a.width = max_pages;
  a.table_in = table_in; a.table_out = table_out; a.free_pages = free_pages;
  a.pool_in = pool_in; a.pool_out = pool_out; a.refs_in = refs_in; a.refs_out = refs_out;
  a.row_off = row_off; a.slots = slot_map; a.slot_rows = slot_rows;
  a.copy_src = copy_src; a.copy_dst = copy_dst; a.status = status;
  a.todo = (int*)workspace; a.last = a.todo + n_pages; a.given = a.last + n_pages; a.copies = a.given + batch;
  a.bad = a.copies + batch;
  launch_pages_plan(a, (hipStream_t)hip_stream);
  HIPCHK(hipGetLastError());
  return ARCHER_OK;
}

size_t archer_pages_compact_ws_bytes(int32_t n_pages) {
  if (n_pages < 1) return 0;
  return align_up(((size_t)n_pages + ((size_t)n_pages + PAGES_BLOCK - 1) / PAGES_BLOCK) * 4, 256);
}

archer_status archer_pages_compact(int32_t batch, const int32_t* len, int32_t page_size, int32_t n_pages, int32_t max_pages,
                                   const int32_t* table_in, int32_t* table_out, const int32_t* refs_in, int32_t* refs_out,
                                   int32_t* free_pages, int32_t* pool_out, int32_t* move_src, int32_t* move_dst,
                                   int32_t* moves, void* workspace, size_t ws_bytes, void* hip_stream) {
  if (!len || !table_in || !table_out || !refs_in || !refs_out || !free_pages || !pool_out || !moves ||
      ((!move_src || !move_dst) && n_pages > 1))
    return archer_fail(ARCHER_E_ARG, "null argument");
  if (batch < 1) return archer_fail(ARCHER_E_SHAPE, "batch must be positive");
  if (const char* e = pages_error(page_size, n_pages)) return archer_fail(ARCHER_E_SHAPE, e);
  if (const char* e = table_error(max_pages, page_size)) return archer_fail(ARCHER_E_SHAPE, e);
  if (overlaps(table_in, table_out, (long long)batch * max_pages) || overlaps(refs_in, refs_out, n_pages))
    return archer_fail(ARCHER_E_ARG, "table_out and refs_out must be table_in and refs_in or not overlap them");
  if (archer_status s = check_workspace(workspace, ws_bytes, archer_pages_compact_ws_bytes(n_pages))) return s;
  PagesCompactArgs a;
  a.batch = batch; a.len = len; a.psh = page_shift(page_size); a.n_pages = n_pages; a.width = max_pages;
  a.table_in = table_in; a.table_out = table_out; a.refs_in = refs_in; a.refs_out = refs_out;
  a.free_pages = free_pages; a.pool_out = pool_out; a.move_src = move_src; a.move_dst = move_dst; a.moves = moves;
  a.rank = (int*)workspace; a.used = a.rank + n_pages;
  launch_pages_compact(a, (hipStream_t)hip_stream);
  HIPCHK(hipGetLastError());
  return ARCHER_OK;
}

archer_status archer_pages_copy(int64_t page_bytes, int32_t n_pages, int32_t n_planes, int64_t plane_stride, void* data,
                                int32_t n, const int32_t* src, const int32_t* dst, const int32_t* count, void* hip_stream) {
  if (page_bytes < 16 || page_bytes % 16 || n_pages < 1) return archer_fail(ARCHER_E_SHAPE, "page_bytes must be a positive multiple of 16, n_pages positive");
  if (page_bytes > INT64_MAX / n_pages) return archer_fail(ARCHER_E_SHAPE, "page_bytes * n_pages must be below 2^63");
  if (n_planes < 1 || plane_stride % 16 || (n_planes > 1 && plane_stride < page_bytes * n_pages))
    return archer_fail(ARCHER_E_SHAPE, "plane_stride must be a multiple of 16, and no less than a plane's bytes");
  if (n < 0) return archer_fail(ARCHER_E_SHAPE, "n must not be negative");
  if (n == 0) return ARCHER_OK;
  if (!data || !src || !dst) return archer_fail(ARCHER_E_ARG, "null argument");
  if ((uintptr_t)data & 15) return archer_fail(ARCHER_E_ARG, "data must be 16-byte aligned");
  PagesCopyArgs a;
  a.data = (char*)data; a.page_bytes = page_bytes; a.plane_stride = plane_stride;
  a.n_pages = n_pages; a.planes = n_planes; a.n = n; a.src = src; a.dst = dst; a.count = count;
  launch_pages_copy(a, (hipStream_t)hip_stream);
  HIPCHK(hipGetLastError());
  return ARCHER_OK;
}

}  // extern "C"
