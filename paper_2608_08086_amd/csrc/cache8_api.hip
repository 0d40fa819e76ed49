// Entry points of the 8-bit paged prompt cache (archer_ops.h): host-side
// checks, then one or two launches.
#include "cache8.h"
#include "paged_api.h"

extern "C" {

size_t archer_cache8_bytes(const archer_cache8* c) {
  if (const char* e = cache_error(c)) {
    archer_fail(c ? ARCHER_E_SHAPE : ARCHER_E_ARG, e);
    return 0;
  }
  return (size_t)c->n_pages * c->n_kv_heads * ((size_t)c->page_size * 2 * c->head_dim + 16);
}

archer_status archer_cache8_write(int32_t dtype, const archer_cache8* cache, int32_t batch, const int32_t* table,
                                  int32_t max_pages, const int32_t* start, const int32_t* row_off, int32_t rows, const void* K,
                                  int64_t k_head, int64_t k_row, const void* V, int64_t v_head, int64_t v_row, int64_t v_dim,
                                  void* hip_stream) {
  archer_status s = check_dtype(dtype);
  if (s || (s = check_cache(cache))) return s;
  if (batch < 1 || batch > 65535) return archer_fail(ARCHER_E_SHAPE, "batch must be in [1, 65535]");
  if (max_pages < 1 || (long long)max_pages * cache->page_size > INT_MAX)
    return archer_fail(ARCHER_E_SHAPE, "max_pages must be positive, max_pages * page_size below 2^31");
  if (rows < 0) return archer_fail(ARCHER_E_SHAPE, "rows must not be negative");
  if (rows == 0) return ARCHER_OK;
  if (!K || !V || !table || !start || !row_off) return archer_fail(ARCHER_E_ARG, "null operand");
  const uintptr_t esz = dtype == ARCHER_BF16 ? 2 : 4;
  if (((uintptr_t)K | (uintptr_t)V) & (esz - 1)) return archer_fail(ARCHER_E_ARG, "K and V must be aligned to their elements");
  if (rows == 1) v_row = 1;      // nothing is a row apart: a view's row stride then says nothing
  if (v_dim != 1 && v_row != 1)
    return archer_fail(ARCHER_E_UNSUPPORTED, "V must have unit stride along its dimensions or along its rows");
  C8WriteArgs a;
  a.c = pool_of(cache);
  a.K = K; a.V = V;
  a.k_head = k_head; a.k_row = k_row; a.v_head = v_head; a.v_row = v_row; a.v_dim = v_dim;
  a.table = table; a.start = start; a.row_off = row_off;
  a.batch = batch; a.width = max_pages; a.rows = rows;
  launch_cache8_write(dtype == ARCHER_FP32, cache->head_dim, a, (hipStream_t)hip_stream);
  HIPCHK(hipGetLastError());
  return ARCHER_OK;
}

archer_status archer_cache8_read(int32_t dtype, const archer_cache8* cache, int32_t rows, const int32_t* slot_map, void* K,
                                 void* V, void* hip_stream) {
  archer_status s = check_dtype(dtype);
  if (s || (s = check_cache(cache))) return s;
  if (rows < 0) return archer_fail(ARCHER_E_SHAPE, "rows must not be negative");
  if (rows == 0) return ARCHER_OK;
  if (!K || !V || !slot_map) return archer_fail(ARCHER_E_ARG, "null operand");
  if (((uintptr_t)K | (uintptr_t)V) & 15) return archer_fail(ARCHER_E_ARG, "K and V must be 16-byte aligned");
  C8ReadArgs a;
  a.c = pool_of(cache);
  a.Ko = K; a.Vo = V; a.slots = slot_map; a.rows = rows;
  launch_cache8_read(dtype == ARCHER_FP32, cache->head_dim, a, (hipStream_t)hip_stream);
  HIPCHK(hipGetLastError());
  return ARCHER_OK;
}

size_t archer_op_attention_cache8_ws_bytes(int32_t dtype, int32_t batch, int32_t G, int32_t Hq, int32_t Hkv, int32_t hd,
                                           int32_t max_cached, int32_t fresh) {
  return attention_ws_bytes(attn8_split, dtype, batch, G, Hq, Hkv, hd, max_cached, fresh);
}

archer_status archer_op_attention_cache8(int32_t dtype, const archer_cache8* cache, int32_t batch, int32_t G, int32_t Hq,
                                         const void* Q, const int32_t* table, int32_t max_pages, const int32_t* cached_len,
                                         int32_t max_cached, const void* K2, const void* Vt2, int32_t ld2,
                                         int32_t fresh_stride, const int32_t* resp_len, void* O, void* workspace,
                                         size_t ws_bytes, void* hip_stream) {
  PagedAttnArgs a;
  if (archer_status s = attention_args(a, attn8_split, dtype, cache, batch, G, Hq, Q, table, max_pages, cached_len, max_cached, K2,
                                       Vt2, ld2, fresh_stride, resp_len, O, workspace, ws_bytes))
    return s;
  launch_attn8(dtype == ARCHER_FP32, a, (hipStream_t)hip_stream);
  HIPCHK(hipGetLastError());
  return ARCHER_OK;
}

}  // extern "C"
