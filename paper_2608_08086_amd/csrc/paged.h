// A paged prompt cache's pool and the arguments of the attention over it, for every format.
#pragma once

#include "common.h"

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));

// pages of a cache
struct PagePool {
  uint8_t* data;
  int n_pages, psh, hkv;     // page size 1 << psh
};

struct PagedAttnArgs {
  PagePool c;
  const void* Q;                // [hq][batch * G][hd]
  const int* table;
  int width;
  const int* cached_len;
  int max_cached;
  const void *K2, *Vt2;         // fresh segment, or null: [hkv][ld2][hd], [hkv][hd][ld2]
  int ld2, fstride;
  const int* resp_len;          // or null
  void* O;                      // [batch * G][hq * hd]
  float *Opart, *ML;            // chunk partials [slots][hkv][G * hq / hkv][hd], and (m, l) of each
  int batch, G, hq, hkv, hd;
  int target, chunk_min, slots, step; // see AttnSplit
  int sorted;                   // row kernel: sequences in the order of falling length
  float scale_log2;
};

// How a call's keys are cut, from what the host knows of it: chunks of
// max(all steps / target, chunk_min) steps, at most `slots` of them (target 0: one per sequence).
struct AttnSplit {
  int target, chunk_min, slots, step;   // step: keys of a step
};
