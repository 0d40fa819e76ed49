// What the entry points of the 4-bit and of the 8-bit prompt cache share: host-side checks of
// a cache and of an attention call over it.
#pragma once

#include <climits>
#include <cmath>
#include <cstring>

#include "archer_ops.h"
#include "errors.h"
#include "host_checks.h"
#include "paged.h"

#define HIPCHK(x)                                                                                              \
  do {                                                                                                         \
    hipError_t e_ = (x);                                                                                       \
    if (e_ != hipSuccess) return archer_fail(ARCHER_E_HIP, std::string(#x) + ": " + hipGetErrorString(e_));    \
  } while (0)

namespace {

// Cache: archer_cache4 or archer_cache8.  Shape checks; data may still be null
template <class Cache> const char* cache_error(const Cache* c) {
  if (!c) return "null cache";
  if (c->head_dim != 64 && c->head_dim != 128) return "head_dim must be 64 or 128";
  if (c->n_kv_heads < 1 || c->n_kv_heads > 65535) return "n_kv_heads must be in [1, 65535]";
  return pages_error(c->page_size, c->n_pages);
}

template <class Cache> archer_status check_cache(const Cache* c) {
  if (const char* e = cache_error(c)) return archer_fail(c ? ARCHER_E_SHAPE : ARCHER_E_ARG, e);
  if (!c->data) return archer_fail(ARCHER_E_ARG, "null cache data");
  if ((uintptr_t)c->data & 15) return archer_fail(ARCHER_E_ARG, "the cache's data must be 16-byte aligned");
  return ARCHER_OK;
}

template <class Cache> PagePool pool_of(const Cache* c) {
  return PagePool{(uint8_t*)c->data, c->n_pages, page_shift(c->page_size), c->n_kv_heads};
}

archer_status check_dtype(int32_t dtype) {
  if (dtype != ARCHER_BF16 && dtype != ARCHER_FP32) return archer_fail(ARCHER_E_ARG, "dtype must be ARCHER_BF16 or ARCHER_FP32");
  return ARCHER_OK;
}

typedef AttnSplit (*SplitFn)(int fp32, int batch, int G, int hq, int hkv, int hd, int max_cached, int fresh);

size_t attention_ws_bytes(SplitFn split, int32_t dtype, int32_t batch, int32_t G, int32_t Hq, int32_t Hkv, int32_t hd,
                          int32_t max_cached, int32_t fresh) {
  if ((dtype != ARCHER_BF16 && dtype != ARCHER_FP32) || batch < 1 || G < 1 || Hkv < 1 || Hq < Hkv || Hq % Hkv || hd < 1 ||
      max_cached < 0)
    return 0;
  const AttnSplit s = split(dtype == ARCHER_FP32, batch, G, Hq, Hkv, hd, max_cached, fresh);
  if (s.slots == batch) return 0;
  const size_t rows = (size_t)s.slots * G * Hq;
  return align_up(rows * hd * 4, 256) + align_up(rows * 2 * 4, 256);
}

// Checks an attention call and makes the kernels' arguments of it.
template <class Cache>
archer_status attention_args(PagedAttnArgs& a, SplitFn split, int32_t dtype, const Cache* cache, int32_t batch, int32_t G,
                             int32_t Hq, const void* Q, const int32_t* table, int32_t max_pages, const int32_t* cached_len,
                             int32_t max_cached, const void* K2, const void* Vt2, int32_t ld2, int32_t fresh_stride,
                             const int32_t* resp_len, void* O, void* workspace, size_t ws_bytes) {
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
  memset(&a, 0, sizeof(a));
  a.c = pool_of(cache);
  a.Q = Q; a.table = table; a.width = max_pages; a.cached_len = cached_len; a.max_cached = max_cached;
  a.K2 = K2; a.Vt2 = Vt2; a.ld2 = ld2; a.fstride = fresh_stride; a.resp_len = resp_len;
  a.O = O;
  a.batch = batch; a.G = G; a.hq = Hq; a.hkv = hkv; a.hd = hd;
  const AttnSplit sp = split(fp32, batch, G, Hq, hkv, hd, max_cached, K2 != nullptr);
  a.target = sp.target; a.chunk_min = sp.chunk_min; a.slots = sp.slots; a.step = sp.step;
  a.scale_log2 = (float)(1.4426950408889634 / std::sqrt((double)hd));
  if (a.slots > batch) {
    if (!workspace || ((uintptr_t)workspace & 255) ||
        ws_bytes < attention_ws_bytes(split, dtype, batch, G, Hq, hkv, hd, max_cached, K2 != nullptr))
      return archer_fail(ARCHER_E_WORKSPACE, "attention workspace too small or misaligned");
    a.Opart = (float*)workspace;
    a.ML = (float*)((char*)workspace + align_up((size_t)a.slots * G * Hq * hd * 4, 256));
  }
  return ARCHER_OK;
}

}  // namespace
