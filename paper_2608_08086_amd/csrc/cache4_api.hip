// Entry points of the 4-bit paged prompt cache (archer_ops.h): host-side
// checks, then one or two launches.
#include <climits>
#include <cmath>
#include <cstring>

#include "archer_ops.h"
#include "cache4.h"
#include "errors.h"

namespace {

#define HIPCHK(x)                                                                                              \
  do {                                                                                                         \
    hipError_t e_ = (x);                                                                                       \
    if (e_ != hipSuccess) return archer_fail(ARCHER_E_HIP, std::string(#x) + ": " + hipGetErrorString(e_));    \
  } while (0)

inline size_t align_up(size_t v, size_t a) { return (v + a - 1) / a * a; }

// log2 of a page size, or -1
int page_shift(int32_t page_size) {
  for (int s = 5; s <= 8; ++s)
    if (page_size == 1 << s) return s;
  return -1;
}

const char* pages_error(int32_t page_size, int32_t n_pages) {
  if (page_shift(page_size) < 0) return "page_size must be 32, 64, 128 or 256";
  if (n_pages < 1 || (long long)n_pages * page_size > INT_MAX) return "n_pages must be positive, n_pages * page_size below 2^31";
  return nullptr;
}

// Shape checks of a cache; data may still be null
const char* cache_error(const archer_cache4* c) {
  if (!c) return "null cache";
  if (c->head_dim != 64 && c->head_dim != 128) return "head_dim must be 64 or 128";
  if (c->n_kv_heads < 1 || c->n_kv_heads > 65535) return "n_kv_heads must be in [1, 65535]";
  return pages_error(c->page_size, c->n_pages);
}

archer_status check_cache(const archer_cache4* c) {
  if (const char* e = cache_error(c)) return archer_fail(c ? ARCHER_E_SHAPE : ARCHER_E_ARG, e);
  if (!c->data) return archer_fail(ARCHER_E_ARG, "null cache data");
  if ((uintptr_t)c->data & 15) return archer_fail(ARCHER_E_ARG, "the cache's data must be 16-byte aligned");
  return ARCHER_OK;
}

C4Pool pool_of(const archer_cache4* c) {
  return C4Pool{(uint8_t*)c->data, c->n_pages, page_shift(c->page_size), c->n_kv_heads};
}

archer_status check_dtype(int32_t dtype) {
  if (dtype != ARCHER_BF16 && dtype != ARCHER_FP32) return archer_fail(ARCHER_E_ARG, "dtype must be ARCHER_BF16 or ARCHER_FP32");
  return ARCHER_OK;
}

}  // namespace

extern "C" {

size_t archer_cache4_bytes(const archer_cache4* c) {
  if (const char* e = cache_error(c)) {
    archer_fail(c ? ARCHER_E_SHAPE : ARCHER_E_ARG, e);
    return 0;
  }
  return (size_t)c->n_pages * c->n_kv_heads * c->page_size * (c->head_dim + c->head_dim / 16);
}

archer_status archer_cache4_plan(int32_t batch, const int32_t* len_old, const int32_t* len_new, int32_t page_size,
                                 int32_t n_pages, int32_t max_pages, int32_t* table, int32_t* free_pages,
                                 const int32_t* pool_in, int32_t* pool_out, int32_t* row_off, int32_t* slot_map,
                                 int32_t slot_rows, int32_t* status, void* hip_stream) {
  if (!len_old || !len_new || !table || !free_pages || !pool_in || !pool_out || !row_off || !status ||
      (!slot_map && slot_rows > 0))
    return archer_fail(ARCHER_E_ARG, "null argument");
  if (batch < 1 || batch > C4_MAX_BATCH) return archer_fail(ARCHER_E_SHAPE, "batch must be in [1, 4096]");
  if (const char* e = pages_error(page_size, n_pages)) return archer_fail(ARCHER_E_SHAPE, e);
  if (max_pages < 1 || (long long)max_pages * page_size > INT_MAX)
    return archer_fail(ARCHER_E_SHAPE, "max_pages must be positive, max_pages * page_size below 2^31");
  if (slot_rows < 0) return archer_fail(ARCHER_E_SHAPE, "slot_rows must not be negative");
  if (pool_in < pool_out + 2 && pool_out < pool_in + 2) return archer_fail(ARCHER_E_ARG, "pool_out must not alias pool_in");
  C4PlanArgs a;
  a.len_old = len_old; a.len_new = len_new;
  a.batch = batch; a.psh = page_shift(page_size); a.n_pages = n_pages; a.width = max_pages;
  a.table = table; a.free_pages = free_pages; a.pool_in = pool_in; a.pool_out = pool_out;
  a.row_off = row_off; a.slots = slot_map; a.status = status; a.slot_rows = slot_rows;
  launch_cache4_plan(a, (hipStream_t)hip_stream);
  HIPCHK(hipGetLastError());
  return ARCHER_OK;
}

archer_status archer_cache4_write(int32_t dtype, const archer_cache4* cache, int32_t rows, const void* K, int64_t k_head,
                                  int64_t k_row, const void* V, int64_t v_head, int64_t v_row, int64_t v_dim,
                                  const int32_t* slot_map, void* hip_stream) {
  archer_status s = check_dtype(dtype);
  if (s || (s = check_cache(cache))) return s;
  if (rows < 0) return archer_fail(ARCHER_E_SHAPE, "rows must not be negative");
  if (rows == 0) return ARCHER_OK;
  if (!K || !V || !slot_map) return archer_fail(ARCHER_E_ARG, "null operand");
  const uintptr_t esz = dtype == ARCHER_BF16 ? 2 : 4;
  if (((uintptr_t)K | (uintptr_t)V) & (esz - 1)) return archer_fail(ARCHER_E_ARG, "K and V must be aligned to their elements");
  if (rows == 1) v_row = 1;      // nothing is a row apart: a view's row stride then says nothing
  if (v_dim != 1 && v_row != 1)
    return archer_fail(ARCHER_E_UNSUPPORTED, "V must have unit stride along its dimensions or along its rows");
  C4RowsArgs a;
  memset(&a, 0, sizeof(a));
  a.c = pool_of(cache);
  a.K = K; a.V = V;
  a.k_head = k_head; a.k_row = k_row; a.v_head = v_head; a.v_row = v_row; a.v_dim = v_dim;
  a.slots = slot_map; a.rows = rows;
  launch_cache4_write(dtype == ARCHER_FP32, cache->head_dim, a, (hipStream_t)hip_stream);
  HIPCHK(hipGetLastError());
  return ARCHER_OK;
}

archer_status archer_cache4_read(int32_t dtype, const archer_cache4* cache, int32_t rows, const int32_t* slot_map, void* K,
                                 void* V, void* hip_stream) {
  archer_status s = check_dtype(dtype);
  if (s || (s = check_cache(cache))) return s;
  if (rows < 0) return archer_fail(ARCHER_E_SHAPE, "rows must not be negative");
  if (rows == 0) return ARCHER_OK;
  if (!K || !V || !slot_map) return archer_fail(ARCHER_E_ARG, "null operand");
  if (((uintptr_t)K | (uintptr_t)V) & 15) return archer_fail(ARCHER_E_ARG, "K and V must be 16-byte aligned");
  C4RowsArgs a;
  memset(&a, 0, sizeof(a));
  a.c = pool_of(cache);
  a.Ko = K; a.Vo = V; a.slots = slot_map; a.rows = rows;
  launch_cache4_read(dtype == ARCHER_FP32, cache->head_dim, a, (hipStream_t)hip_stream);
  HIPCHK(hipGetLastError());
  return ARCHER_OK;
}

size_t archer_op_attention_cache4_ws_bytes(int32_t dtype, int32_t batch, int32_t G, int32_t Hq, int32_t Hkv, int32_t hd,
                                           int32_t max_cached, int32_t fresh) {
  if ((dtype != ARCHER_BF16 && dtype != ARCHER_FP32) || batch < 1 || G < 1 || Hkv < 1 || Hq < Hkv || Hq % Hkv || hd < 1 ||
      max_cached < 0)
    return 0;
  const Attn4Split s = attn4_split(dtype == ARCHER_FP32, batch, G, Hq, Hkv, hd, max_cached, fresh);
  if (s.slots == batch) return 0;
  const size_t rows = (size_t)s.slots * G * Hq;
  return align_up(rows * hd * 4, 256) + align_up(rows * 2 * 4, 256);
}

archer_status archer_op_attention_cache4(int32_t dtype, const archer_cache4* cache, int32_t batch, int32_t G, int32_t Hq,
                                         const void* Q, const int32_t* table, int32_t max_pages, const int32_t* cached_len,
                                         int32_t max_cached, const void* K2, const void* Vt2, int32_t ld2,
                                         int32_t fresh_stride, const int32_t* resp_len, void* O, void* workspace,
                                         size_t ws_bytes, void* hip_stream) {
  archer_status s = check_dtype(dtype);
  if (s || (s = check_cache(cache))) return s;
  if (!Q || !table || !cached_len || !O) return archer_fail(ARCHER_E_ARG, "null operand");
  if (!K2 != !Vt2) return archer_fail(ARCHER_E_ARG, "K2 and Vt2 must both be given, or neither");
  const int hkv = cache->n_kv_heads, hd = cache->head_dim;
  if (batch < 1 || batch > 65535 || G < 1) return archer_fail(ARCHER_E_SHAPE, "batch must be in [1, 65535] and G positive");
  if (Hq < 1 || Hq % hkv) return archer_fail(ARCHER_E_SHAPE, "Hq must be a multiple of the cache's heads");
  if (max_pages < 1 || (long long)max_pages * cache->page_size > INT_MAX || max_cached < 0)
    return archer_fail(ARCHER_E_SHAPE, "bad max_pages or max_cached");
  if ((long long)batch * G > INT_MAX || (long long)batch * G * Hq > INT_MAX)
    return archer_fail(ARCHER_E_SHAPE, "batch * G * Hq must be below 2^31");
  if (K2 && (ld2 % 8 || fresh_stride % 8 || fresh_stride < G || (long long)batch * fresh_stride > ld2))
    return archer_fail(ARCHER_E_SHAPE, "bad fresh segment: ld2 and fresh_stride multiples of 8, fresh_stride >= G, batch * fresh_stride <= ld2");
  if (((uintptr_t)Q | (uintptr_t)K2 | (uintptr_t)Vt2 | (uintptr_t)O) & 15)
    return archer_fail(ARCHER_E_ARG, "Q, K2, Vt2 and O must be 16-byte aligned");
  const int fp32 = dtype == ARCHER_FP32;
  Attn4Args a;
  memset(&a, 0, sizeof(a));
  a.c = pool_of(cache);
  a.Q = Q; a.table = table; a.width = max_pages; a.cached_len = cached_len; a.max_cached = max_cached;
  a.K2 = K2; a.Vt2 = Vt2; a.ld2 = ld2; a.fstride = fresh_stride; a.resp_len = resp_len;
  a.O = O;
  a.batch = batch; a.G = G; a.hq = Hq; a.hkv = hkv; a.hd = hd;
  const Attn4Split sp = attn4_split(fp32, batch, G, Hq, hkv, hd, max_cached, K2 != nullptr);
  a.target = sp.target; a.chunk_min = sp.chunk_min; a.slots = sp.slots; a.step = sp.step;
  a.scale_log2 = (float)(1.4426950408889634 / std::sqrt((double)hd));
  if (a.slots > batch) {
    if (!workspace || ((uintptr_t)workspace & 255) ||
        ws_bytes < archer_op_attention_cache4_ws_bytes(dtype, batch, G, Hq, hkv, hd, max_cached, K2 != nullptr))
      return archer_fail(ARCHER_E_WORKSPACE, "attention workspace too small or misaligned");
    a.Opart = (float*)workspace;
    a.ML = (float*)((char*)workspace + align_up((size_t)a.slots * G * Hq * hd * 4, 256));
  }
  if (launch_attn4(fp32, a, (hipStream_t)hip_stream)) return archer_fail(ARCHER_E_UNSUPPORTED, "attention shape unsupported");
  HIPCHK(hipGetLastError());
  return ARCHER_OK;
}

}  // extern "C"
