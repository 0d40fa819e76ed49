// The 8-bit paged prompt cache: layout, kernel arguments and launchers.
//
// A stored element is an e4m3 value (sign, four exponent bits, three mantissa
// bits, at most 448) times a power of two that the 32 tokens of a block share, for a
// head's keys and for its values.  gfx950 expands two such elements to fp16
// or fp32, scale included, in one instruction, and with the scale's exponent in [-15, 7]
// every stored element is exact in fp16 (2^-24 ... 57344).
//
// The bytes of one head's share of a page of T tokens (D = head_dim):
//   keys    [T][D]
//   values  [T/8][D/32][16][2][8]   8-token blocks: dimension u D/16 + 2 i + s of token t at [i][u][s][t]
//   scales  [T/32][2], 16 bytes     biased exponents of a block's keys and of its values
// A lane of the score MFMA reads 16-byte pieces of one key's row; a lane of the P V MFMA
// needs 8 keys of one dimension, which are 8 consecutive bytes here, and a piece of 16
// bytes is two of its dimensions.  No two tokens share a byte, but a block's tokens share
// its scale: a block is stored by one workgroup.
#pragma once

#include "paged.h"

constexpr int C8_EMIN = 112, C8_EMAX = 134;   // biased scale exponents: 2^-15 .. 2^7
constexpr int C8_BLOCK = 32;                  // tokens of a scale

template <int HD> struct C8 {
  static constexpr int VBLK = 8 * HD;         // bytes of an 8-token block of values
  __host__ __device__ static size_t page_bytes(int T) { return (size_t)T * (2 * HD) + 16; }
  __device__ static int voff(int T) { return T * HD; }
  __device__ static int soff(int T) { return 2 * T * HD; }
};

struct C8WriteArgs {
  PagePool c;
  const void *K, *V;            // sources (strides in elements)
  long k_head, k_row, v_head, v_row, v_dim;
  const int *table, *start, *row_off;
  int batch, width, rows;
};

struct C8ReadArgs {
  PagePool c;
  void *Ko, *Vo;                // [hkv][rows][hd]
  const int* slots;
  int rows;
};

void launch_cache8_write(int fp32, int hd, const C8WriteArgs& a, hipStream_t st);
void launch_cache8_read(int fp32, int hd, const C8ReadArgs& a, hipStream_t st);
AttnSplit attn8_split(int fp32, int batch, int G, int hq, int hkv, int hd, int max_cached, int fresh);
void launch_attn8(int fp32, const PagedAttnArgs& a, hipStream_t st);
