// The 4-bit paged prompt cache: layout, kernel arguments and launchers.
//
// A stored element is an e2m1 value (sign, two exponent bits, one mantissa
// bit: 0, .5, 1, 1.5, 2, 3, 4, 6) times a power of two that 32 consecutive
// dimensions of one key or value share.  gfx950 expands two such elements to
// fp16 or fp32, scale included, in one full-rate instruction (measured: 505 G
// wave instructions/s, the rate of an fma), and with the scale's exponent in
// [-23, 13] every stored element is exact in fp16 (2^-24 ... 49152).
//
// The bytes of one head's share of a page of T tokens (D = head_dim):
//   keys    [T][D/2]                  byte j: dimensions 2j (low nibble), 2j + 1
//   values  [T/8][16][8][D/32]        8-token blocks of 16 units of D/16 dimensions, tokens inside
//   key scales, value scales [T/8][D/32][8]   biased exponents, tokens inside
// A key's row is what a lane of the score MFMA reads (32 or 16 consecutive
// dimensions of one key).  A lane of the P V MFMA needs 8 keys of one
// dimension: the value unit of an 8-token block gives it D/16 dimensions of 8
// keys in 16 or 32 consecutive bytes, to be transposed in registers; no two
// tokens share a byte, so tokens are stored without read-modify-write.
#pragma once

#include "common.h"

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));

constexpr int C4_EMIN = 104, C4_EMAX = 140;   // biased scale exponents: 2^-23 .. 2^13
constexpr int C4_NAN = 255;                   // scale byte of a block that holds a NaN
constexpr int C4_MAX_BATCH = 4096;            // requests of one plan (LDS: three prefix arrays)

template <int HD> struct C4 {
  static constexpr int KROW = HD / 2;                    // bytes of a key
  static constexpr int VUNIT = 8 * HD / 32;              // bytes of a value unit (8 tokens)
  static constexpr int VBLK = 16 * VUNIT;                // bytes of a value block
  static constexpr int SBLK = HD / 32 * 8;               // scale bytes of an 8-token block
  __host__ __device__ static size_t page_bytes(int T) { return (size_t)T * (HD + HD / 16); }
  __device__ static int voff(int T) { return T * KROW; }
  __device__ static int ksoff(int T) { return T * HD; }
  __device__ static int vsoff(int T) { return T * HD + T * (HD / 32); }
};

struct C4Pool {
  uint8_t* data;
  int n_pages, psh, hkv;     // page size 1 << psh
};

struct C4PlanArgs {
  const int *len_old, *len_new;
  int batch, psh, n_pages, width;   // width: entries of a table row
  int *table, *free_pages;
  const int* pool_in;
  int *pool_out, *row_off, *slots, *status;
  int slot_rows;
};

struct C4RowsArgs {
  C4Pool c;
  const void *K, *V;            // write: sources (strides in elements); read: unused
  long k_head, k_row, v_head, v_row, v_dim;
  void *Ko, *Vo;                // read: [hkv][rows][hd]
  const int* slots;
  int rows;
};

struct Attn4Args {
  C4Pool c;
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
  int target, chunk_min, slots, step; // see Attn4Split
  int sorted;                   // row kernel: sequences in the order of falling length
  float scale_log2;
};

// How a call's keys are cut, from what the host knows of it: chunks of
// max(all steps / target, chunk_min) steps, at most `slots` of them (target 0: one per sequence).
struct Attn4Split {
  int target, chunk_min, slots, step;   // step: keys of a step
};

void launch_cache4_plan(const C4PlanArgs& a, hipStream_t st);
int launch_cache4_write(int fp32, int hd, const C4RowsArgs& a, hipStream_t st);
int launch_cache4_read(int fp32, int hd, const C4RowsArgs& a, hipStream_t st);
Attn4Split attn4_split(int fp32, int batch, int G, int hq, int hkv, int hd, int max_cached, int fresh);
int launch_attn4(int fp32, const Attn4Args& a, hipStream_t st);
