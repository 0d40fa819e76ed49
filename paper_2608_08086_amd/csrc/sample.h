// Sampling of a token per row of logits: kernel arguments and launcher.
#pragma once

#include "common.h"

constexpr int SAMPLE_MAX_VOCAB = 1 << 19;   // 2^19 fixed-point weights of 2^44 fit 64 bits

struct SampleArgs {
  const void* logits;
  long ld;                      // elements from row to row
  int rows, vocab, exclude;     // exclude: a token that is never drawn, or -1
  const float* u;
  const float* temperature;     // [rows], or null: 1
  const int* top_k;             // [rows], or null: off
  const float *top_p, *min_p;
  int* token;
  float* logp;                  // or null
};

size_t sample_ws_bytes(int rows);
void launch_sample(int dtype, const SampleArgs& a, void* workspace, hipStream_t st);
