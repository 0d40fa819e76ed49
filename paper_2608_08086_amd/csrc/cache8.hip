// Kernels that store rows of keys and values in the 8-bit prompt cache and read them
// back (layout: cache8.h).
//
// Store.  Rows are given by their sequences: rows row_off[b] .. row_off[b + 1] - 1 are the
// tokens from position start[b] on of the sequence whose pages row b of the table lists.  So a
// block of 32 tokens has one workgroup, whatever part of it is stored:
//   top = max |x| of its new rows, over the head's dimensions
//   2^e   e the least integer with top <= 448 * 2^e, clamped to [-15, 7]; of a block that holds earlier
//         tokens of the sequence no less than theirs, and they are re-expressed with it
//   code  nearest e4m3 value of x / 2^e, ties to the even code; saturates where e is clamped
// and the whole block is written (zeros behind the last row).  All of it is exact in fp32 but
// the rounding, which is the hardware's own conversion.
//
// What bounds them: memory.  21500 rows of 32 heads of 128 in fp16, with pages of 64: the keys are stored in 60 us (4.4 TB/s of
// rows and codes), the transposed values in 62, all are read back in 111 (4.8 TB/s).
#include <algorithm>
#include <climits>

#include "cache8.h"

namespace {

constexpr int NT = 256;
constexpr int UNIT = 2 * C8_BLOCK;          // tokens of a storing workgroup
constexpr int LONG_UNIT = 128;              // of one that stores transposed values: the consecutive ones that it reads of a dimension

typedef short i16x2 __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// inclusive sum over the wave's lanes
__device__ __forceinline__ int wave_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);      // row_shr 1, 2, 4, 8, row_bcast 15, 31
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
  return x;
}

// The batch's units of U tokens, in sequence order: unit `key` is unit `first` + n of sequence b.
struct Span {
  int b, start, row0, row1, unit;   // rows row0 .. row1 - 1 at positions start ..; unit: number of the U tokens
};
template <int U> __device__ __forceinline__ Span find_unit(const C8WriteArgs& a, int key) {
  const int lane = threadIdx.x & 63;
  int base = 0;
  for (int b0 = 0; b0 < a.batch; b0 += 64) {
    const int b = min(b0 + lane, a.batch - 1);
    // rows outside the arrays are none: neither is a sequence that does not fit the table
    const int s = a.start[b], r0 = min(max(a.row_off[b], 0), a.rows), r1 = min(max(a.row_off[b + 1], r0), a.rows);
    const long long cap = (long long)a.width << a.c.psh;
    const int fit = s < 0 ? 0 : (int)min((long long)(r1 - r0), max(cap - s, 0LL));
    const int n = b0 + lane < a.batch && fit > 0 ? (int)(((long long)s + fit - 1) / U) - s / U + 1 : 0;
    const int incl = wave_scan(n);
    const unsigned long long m = __ballot(base + incl > key);
    if (m) {
      const int at = __ffsll(m) - 1;
      Span v;
      v.b = b0 + at;
      v.start = __builtin_amdgcn_readlane(s, at);
      v.row0 = __builtin_amdgcn_readlane(r0, at);
      v.row1 = v.row0 + __builtin_amdgcn_readlane(fit, at);
      v.unit = v.start / U + key - (base + __builtin_amdgcn_readlane(incl - n, at));
      return v;
    }
    base += __builtin_amdgcn_readlane(incl, 63);
  }
  return Span{-1, 0, 0, 0, 0};
}

__device__ __forceinline__ float scale_of(unsigned eb) { return __uint_as_float(eb << 23); }

// the smallest biased exponent that reaches top (its bits)
__device__ __forceinline__ unsigned exponent_of(unsigned top) {
  const unsigned e = (top + 0x1fffffu) >> 23;     // 1.m 2^E: one more when 1.m > 1.75
  return min(max(e, (unsigned)C8_EMIN + 8u), (unsigned)C8_EMAX + 8u) - 8u;
}

// four codes
__device__ __forceinline__ unsigned pack4(const float* x, float sc) {
  i16x2 r = {0, 0};
  r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, x[0], x[1], sc, false);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, x[2], x[3], sc, true);
  return __builtin_bit_cast(unsigned, r);
}
__device__ __forceinline__ void unpack4(float* x, unsigned c, float sc) {
  const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c, sc, false), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c, sc, true);
  x[0] = a[0]; x[1] = a[1]; x[2] = b[0]; x[3] = b[1];
}

// N consecutive elements, aligned to an element
template <int N, class T> __device__ __forceinline__ void load_n(T (&x)[N], const T* p) { __builtin_memcpy(x, p, N * sizeof(T)); }

// A workgroup's two blocks.
//   keys     thread: row tid / 8 of each block, HD / 8 dimensions from (tid % 8) HD / 8
//   values   wave w: 8-token block w of each block; lane (of HD / 2): dimensions 2 lane, 2 lane + 1
template <class T, int HD, int KIND>     // 0 keys, 1 values
__device__ __forceinline__ void write_unit(const C8WriteArgs& a, const Span& v, int h) {
  using L = C8<HD>;
  constexpr int E = HD / 8, NB = UNIT / C8_BLOCK;       // elements of a thread of a block (values: 16, of fewer threads)
  constexpr int EV = KIND == 0 ? E : 16;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, Tp = 1 << a.c.psh;
  const T* src = KIND == 0 ? (const T*)a.K + h * a.k_head : (const T*)a.V + h * a.v_head;
  const bool on = KIND == 0 || HD == 128 || lane < HD / 2;
  // a thread's 8-token block and first dimension of its pair (values)
  const int tb = w, dim = KIND == 0 ? (tid & 7) * E : 2 * min(lane, HD / 2 - 1);
  const int n = v.row1 - v.row0, end = v.start + n;
  float x[NB][EV];
  unsigned top[NB], old[NB];          // old: scale byte of a block that is joined, else 0
  uint8_t* page[NB];
  int at[NB];
#pragma unroll
  for (int k = 0; k < NB; ++k) {
    const int p0 = v.unit * UNIT + k * C8_BLOCK, j = min(p0 >> a.c.psh, a.width - 1);
    const int pg = a.table[(size_t)v.b * a.width + j];
    const bool ok = pg >= 0 && pg < a.c.n_pages && p0 < end && p0 + C8_BLOCK > v.start;
    page[k] = ok ? a.c.data + ((size_t)pg * a.c.hkv + h) * L::page_bytes(Tp) : nullptr;
    at[k] = p0 & (Tp - 1);
  }
  // every block's rows are requested before the first is looked at; rows that are not the
  // sequence's read its first or last one
  T t[NB][EV];
#pragma unroll
  for (int k = 0; k < NB; ++k) {
    const int p0 = v.unit * UNIT + k * C8_BLOCK;
    auto row = [&](int i) __attribute__((always_inline)) { return (long)v.row0 + min(max(p0 + i - v.start, 0), n - 1); };
    if constexpr (KIND == 0) {
      load_n<EV>(t[k], src + row(tid >> 3) * a.k_row + dim);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        T y[2];
        load_n<2>(y, src + row(8 * tb + i) * a.v_row + dim);
        t[k][i] = y[0];
        t[k][8 + i] = y[1];
      }
    }
  }
  // token of element e of this thread
  auto token = [&](int e) __attribute__((always_inline)) { return KIND == 0 ? tid >> 3 : 8 * tb + (e & 7); };
  const int off = KIND == 0 ? (tid >> 3) * HD + dim
                            : L::voff(Tp) + tb * L::VBLK + (dim % (HD / 16)) / 2 * 256 + dim / (HD / 16) * 16;
  // a block that is joined: its earlier tokens and their scale, before the barrier after which they are written
  unsigned was[NB][EV / 4];
  uint8_t *scale[NB], *dst[NB];
#pragma unroll
  for (int k = 0; k < NB; ++k) {
    scale[k] = page[k] + L::soff(Tp) + (at[k] >> 5) * 2 + (KIND != 0);
    dst[k] = page[k] + (size_t)at[k] * HD + off;      // (values: 32 tokens are 4 VBLK = 32 HD bytes as well)
    old[k] = 0;
    if (page[k] && v.unit * UNIT + k * C8_BLOCK < v.start) {
      old[k] = *scale[k];
      if (on) __builtin_memcpy(was[k], __builtin_assume_aligned(dst[k], EV), EV);
    }
  }
  __shared__ unsigned red[NB][NT / 64];
#pragma unroll
  for (int k = 0; k < NB; ++k) {
    const int p0 = v.unit * UNIT + k * C8_BLOCK;
    float m = 0.f;
#pragma unroll
    for (int e = 0; e < EV; ++e) {
      const int p = p0 + token(e);
      x[k][e] = on && p >= v.start && p < end ? to_f32(t[k][e]) : 0.f;
      m = fmaxf(m, fabsf(x[k][e]));       // a NaN is no maximum
    }
    top[k] = __float_as_uint(wave_max(m));
    if (lane == 0) red[k][w] = top[k];
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < NB; ++k) {
    if (!page[k]) continue;
    const int p0 = v.unit * UNIT + k * C8_BLOCK;
    unsigned m = 0;
#pragma unroll
    for (int i = 0; i < NT / 64; ++i) m = max(m, red[k][i]);
    unsigned eb = exponent_of(m);
    if (p0 < v.start) {
      const unsigned e = min(max(old[k], (unsigned)C8_EMIN), (unsigned)C8_EMAX);
      eb = max(eb, e);
#pragma unroll
      for (int e4 = 0; e4 < EV; e4 += 4) {
        float y[4];
        unpack4(y, on ? was[k][e4 / 4] : 0u, scale_of(e));
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (p0 + token(e4 + i) < v.start) x[k][e4 + i] = y[i];
      }
    }
    if (eb == (unsigned)C8_EMAX) {        // only here can an element lie beyond 448
      const float most = 448.f * scale_of(eb);
#pragma unroll
      for (int e = 0; e < EV; ++e) x[k][e] = x[k][e] > most ? most : x[k][e] < -most ? -most : x[k][e];
    }
    unsigned c[EV / 4];
#pragma unroll
    for (int e = 0; e < EV; e += 4) c[e / 4] = pack4(&x[k][e], scale_of(eb));
    if (on) __builtin_memcpy(__builtin_assume_aligned(dst[k], EV), c, EV);
    if (tid == 0) *scale[k] = (uint8_t)eb;
  }
}

template <class T, int HD>
__global__ __launch_bounds__(NT) void cache8_write_kernel(C8WriteArgs a) {
  const Span v = find_unit<UNIT>(a, blockIdx.x);
  if (v.b < 0) return;
  if (blockIdx.z == 0) write_unit<T, HD, 0>(a, v, blockIdx.y);
  else write_unit<T, HD, 1>(a, v, blockIdx.y);
}

// Two dimensions of 8 tokens.  `in`: all ones in the halves of tokens that count, two a word.
template <class T> struct Pair {
  float x[16];
  __device__ __forceinline__ void load(int s, const float* p) { __builtin_memcpy(&x[8 * s], p, 32); }
  __device__ __forceinline__ void set(int e, float y) { x[e] = y; }
  static __device__ __forceinline__ bool has(const unsigned (&in)[4], int e) { return in[e % 8 / 2] >> (e % 2 * 16) & 1; }
  __device__ __forceinline__ void keep(const unsigned (&in)[4]) {
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = has(in, e) ? x[e] : 0.f;
  }
  __device__ __forceinline__ float largest() const {       // of |x|; a NaN is none
    float m = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) m = fmaxf(m, fabsf(x[e]));
    return m;
  }
  __device__ __forceinline__ void join(const unsigned (&c)[4], float sc, const unsigned (&in)[4]) {      // stored tokens
#pragma unroll
    for (int e = 0; e < 16; e += 4) {
      float y[4];
      unpack4(y, c[e / 4], sc);
#pragma unroll
      for (int j = 0; j < 4; ++j) x[e + j] = has(in, e + j) ? y[j] : x[e + j];
    }
  }
  __device__ __forceinline__ void clamp(float most) {
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = x[e] > most ? most : x[e] < -most ? -most : x[e];
  }
  __device__ __forceinline__ u32x4 codes(float sc) const { return u32x4{pack4(x, sc), pack4(x + 4, sc), pack4(x + 8, sc), pack4(x + 12, sc)}; }
};
// in fp16 two elements to an instruction; every stored element is one of fp16
template <> struct Pair<f16> {
  unsigned x[8];
  static __device__ __forceinline__ unsigned bits(f16 y) { return __builtin_bit_cast(unsigned short, y); }
  __device__ __forceinline__ void load(int s, const f16* p) { __builtin_memcpy(&x[4 * s], p, 16); }
  __device__ __forceinline__ void set(int e, f16 y) { x[e / 2] = e % 2 ? x[e / 2] | bits(y) << 16 : bits(y); }      // (in order)
  __device__ __forceinline__ void keep(const unsigned (&in)[4]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] &= in[i % 4];
  }
  __device__ __forceinline__ float largest() const {
    u16x2 m = {0, 0};                      // the bits of |x| are ordered as it is, NaNs above all
#pragma unroll
    for (int i = 0; i < 8; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, x[i] & 0x7fff7fffu));
    unsigned t = max(m[0], m[1]);
    if (__ballot(t > 0x7c00)) {
      t = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 32; j += 16) {
          const unsigned y = x[i] >> j & 0x7fff;
          t = y <= 0x7c00 ? max(t, y) : t;
        }
    }
    return (float)__builtin_bit_cast(f16, (unsigned short)t);
  }
  __device__ __forceinline__ void join(const unsigned (&c)[4], float sc, const unsigned (&in)[4]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const f16x2 y = i % 2 ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c[i / 2], sc, true) : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c[i / 2], sc, false);
      x[i] = (x[i] & ~in[i % 4]) | (__builtin_bit_cast(unsigned, y) & in[i % 4]);
    }
  }
  __device__ __forceinline__ void clamp(float most) {      // (most is 448 * 2^7 = 57344)
    const unsigned top = bits((f16)most);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      unsigned y = 0;
#pragma unroll
      for (int j = 0; j < 32; j += 16) {
        const unsigned v = x[i] >> j & 0xffff, m = v & 0x7fff;
        y |= (m <= 0x7c00 && m > top ? (v & 0x8000) | top : v) << j;
      }
      x[i] = y;
    }
  }
  __device__ __forceinline__ u32x4 codes(float sc) const {
    u32x4 c;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      i16x2 r = {0, 0};
      r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(r, __builtin_bit_cast(f16x2, x[2 * i]), sc, false);
      r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(r, __builtin_bit_cast(f16x2, x[2 * i + 1]), sc, true);
      c[i] = __builtin_bit_cast(unsigned, r);
    }
    return c;
  }
};

// Transposed values.  A wave has HD / waves dimensions, two groups of two a lane; lane l 8-token block l % BLOCKS, so that
// BLOCKS lanes read the unit's tokens of a dimension.  Codes go by LDS, as a lane's 16 bytes are apart from the next one's.
// (The time goes with the instructions: 106 us where every element was widened to fp32 and the codes' places were found per
// lane.  Units of 64 tokens and no LDS 125 us, of 256 tokens 129.)
template <class T, int HD>
__global__ __launch_bounds__(LONG_UNIT * 4) void cache8_write_long_kernel(C8WriteArgs a) {
  using L = C8<HD>;
  constexpr int LNT = LONG_UNIT * 4, NW = LNT / 64, BLOCKS = LONG_UNIT / 8, SCALES = LONG_UNIT / C8_BLOCK;
  constexpr int NI = HD / 64;                            // items of a thread: two dimensions of 8 tokens
  constexpr int PITCH = L::VBLK + 16;
  __shared__ unsigned red[SCALES][NW];
  __shared__ alignas(16) uint8_t tile[BLOCKS * PITCH];
  const Span v = find_unit<LONG_UNIT>(a, blockIdx.x);
  if (v.b < 0) return;
  const int h = blockIdx.y, tid = threadIdx.x, lane = tid & 63, w = tid >> 6, Tp = 1 << a.c.psh;
  const T* src = (const T*)a.V + h * a.v_head;
  const int tb = lane % BLOCKS, n = v.row1 - v.row0, end = v.start + n, u0 = v.unit * LONG_UNIT, p = u0 + tb * 8, q = p - v.start;
  auto dim = [&](int i) __attribute__((always_inline)) { return HD / NW * w + 2 * (NI * (lane / BLOCKS) + i); };
  // every row is requested before the first is looked at; rows that are not the sequence's read its first or last one
  Pair<T> t[NI];
#pragma unroll
  for (int i = 0; i < NI; ++i) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const T* from = src + (dim(i) + s) * a.v_dim + v.row0;
      if (q >= 0 && q + 8 <= n) {
        t[i].load(s, from + q);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) t[i].set(8 * s + j, from[min(max(q + j, 0), n - 1)]);
      }
    }
  }
  // where block k of the unit is, or null
  auto head = [&](int k) __attribute__((always_inline)) -> uint8_t* {
    const int p0 = u0 + k * C8_BLOCK, pg = a.table[(size_t)v.b * a.width + min(p0 >> a.c.psh, a.width - 1)];
    const bool ok = pg >= 0 && pg < a.c.n_pages && p0 < end && p0 + C8_BLOCK > v.start;
    return ok ? a.c.data + ((size_t)pg * a.c.hkv + h) * L::page_bytes(Tp) : nullptr;
  };
  const int k = tb / 4, p0 = u0 + k * C8_BLOCK;          // the lane's block of a scale
  uint8_t* const page = head(k);
  uint8_t* const scale = page + L::soff(Tp) + ((p0 & (Tp - 1)) >> 5) * 2 + 1;
  unsigned old = 0;                                      // scale byte of a block that is joined
  if (page && p0 < v.start) old = min(max((unsigned)*scale, (unsigned)C8_EMIN), (unsigned)C8_EMAX);
  auto tokens = [&](int from, int to, unsigned (&in)[4]) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int at = p + 2 * j;
      in[j] = (at >= from && at < to ? 0xffffu : 0u) | (at + 1 >= from && at + 1 < to ? 0xffff0000u : 0u);
    }
  };
  if (u0 < v.start || u0 + LONG_UNIT > end) {
    unsigned in[4];
    tokens(v.start, end, in);
#pragma unroll
    for (int i = 0; i < NI; ++i) t[i].keep(in);
  }
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < NI; ++i) m = fmaxf(m, t[i].largest());
#pragma unroll
  for (int o = 1; o < 64; o = o == 2 ? BLOCKS : 2 * o) m = fmaxf(m, __shfl_xor(m, o, 64));      // over the block's lanes
  if (lane < BLOCKS && lane % 4 == 0) red[k][w] = __float_as_uint(m);
  __syncthreads();                                       // (scales are read before they are written, too)
  unsigned top = 0;
#pragma unroll
  for (int j = 0; j < NW; ++j) top = max(top, red[k][j]);
  const unsigned eb = max(exponent_of(top), old);
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int off = dim(i) % (HD / 16) / 2 * 256 + dim(i) / (HD / 16) * 16;
    if (old) {
      unsigned c[4], in[4];
      __builtin_memcpy(c, __builtin_assume_aligned(page + L::voff(Tp) + ((p & (Tp - 1)) >> 3) * L::VBLK + off, 16), 16);
      tokens(INT_MIN, v.start, in);
      t[i].join(c, scale_of(old), in);
    }
    if (eb == (unsigned)C8_EMAX) t[i].clamp(448.f * scale_of(eb));      // only here can an element lie beyond 448
    *(u32x4*)(tile + tb * PITCH + off) = t[i].codes(scale_of(eb));
  }
  if (page && w == 0 && lane < BLOCKS && lane % 4 == 0) *scale = (uint8_t)eb;
  __syncthreads();
  constexpr int PIECES = L::VBLK / 16;
#pragma unroll
  for (int i = tid; i < BLOCKS * PIECES; i += LNT) {
    const int b = i / PIECES, piece = i % PIECES * 16;
    uint8_t* to = head(__builtin_amdgcn_readfirstlane(b / 4));      // (64 / PIECES 8-token blocks of a wave)
    if (to) *(u32x4*)(to + L::voff(Tp) + (((u0 + b * 8) & (Tp - 1)) >> 3) * L::VBLK + piece) = *(const u32x4*)(tile + b * PITCH + piece);
  }
}

// Read back.  A slot outside the cache gives zeros.
//   keys    a thread 8 dimensions of a row
//   values  8 rows of HD / 2 lanes, two dimensions each.  Where the slots follow each other in one page, the
//           codes are those of two 8-token blocks at most, 16 bytes a lane each: shifted to begin at the first row,
//           two dimensions' codes of a row side by side.  Else byte by byte (all of them: 165 us with the keys, not 111).
template <class T> __device__ __forceinline__ void put2(T* out, unsigned c, bool high, float sc) {      // (its low or high half)
  if constexpr (sizeof(T) == 2) {
    const f16x2 y = high ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c, sc, true) : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c, sc, false);
    *(unsigned*)out = __builtin_bit_cast(unsigned, y);
  } else {
    *(f32x2*)out = high ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c, sc, true) : __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c, sc, false);
  }
}
template <class T, int HD> __device__ __forceinline__ void read_values(const C8ReadArgs& a, long r0, int h) {
  using L = C8<HD>;
  constexpr int G = HD / 2, VF = HD / 16;                  // lanes of 8 rows
  const int lane = threadIdx.x & 63, p = lane % G, j = lane & 7, T_ = 1 << a.c.psh;
  r0 += lane / G * 8;
  const long all = (long)a.c.n_pages << a.c.psh;
  const int slot = a.slots[min(r0 + j, (long)a.rows - 1)], first = __shfl(slot, lane - p, 64), t0 = first & (T_ - 1);
  const bool follows = (long)slot == (long)first + j && first >= 0 && first + 7L < all && t0 + 7 < T_ && r0 + 7 < a.rows;
  const bool run = (__ballot(follows) >> (lane - p) & 0xff) == 0xff;
  const int d = 2 * p, off = d % VF / 2 * 256 + d / VF * 16;      // of the lane's two dimensions in an 8-token block
  auto head = [&](int s) __attribute__((always_inline)) { return a.c.data + ((size_t)(s >> a.c.psh) * a.c.hkv + h) * L::page_bytes(T_); };
  T* out = (T*)a.Vo + ((size_t)h * a.rows + r0) * HD + d;
  if (run) {
    const uint8_t* page = head(first);
    const uint8_t* codes = page + L::voff(T_) + (t0 >> 3) * L::VBLK + off;
    u32x4 lo = *(const u32x4*)codes, hi = lo;
    const int o = t0 & 7;
    if (o) hi = *(const u32x4*)(codes + L::VBLK);
    unsigned c[4];                                         // tokens 0 .. 3 of either dimension, then 4 .. 7
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      unsigned long long x = (unsigned long long)lo[2 * s + 1] << 32 | lo[2 * s];
      const unsigned long long y = (unsigned long long)hi[2 * s + 1] << 32 | hi[2 * s];
      if (o) x = x >> (8 * o) | y << (64 - 8 * o);
      c[s] = (unsigned)x;
      c[2 + s] = (unsigned)(x >> 32);
    }
    const uint8_t* scales = page + L::soff(T_) + 1;
    const float s0 = scale_of(scales[(t0 >> 5) * 2]), s1 = scale_of(scales[((t0 + 7) >> 5) * 2]);
    const int more = 32 - (t0 & 31);                       // rows of the first scale
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      // (dimension 0, dimension 1) of two rows
      const unsigned y = __builtin_amdgcn_perm(c[i / 4 * 2 + 1], c[i / 4 * 2], i % 4 ? 0x07030602u : 0x05010400u);
      put2(out + (size_t)i * HD, y, false, i < more ? s0 : s1);
      put2(out + (size_t)(i + 1) * HD, y, true, i + 1 < more ? s0 : s1);
    }
    return;
  }
  // every row's bytes are requested before the first is stored
  unsigned y[8];
  float sc[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int s = __shfl(slot, lane - p + i, 64);
    const bool ok = s >= 0 && s < all;
    const int t = ok ? s & (T_ - 1) : 0;
    const uint8_t* page = head(ok ? s : 0);
    const uint8_t* codes = page + L::voff(T_) + (t >> 3) * L::VBLK + off + (t & 7);
    y[i] = ok ? codes[0] | (unsigned)codes[8] << 8 : 0u;
    sc[i] = scale_of(ok ? page[L::soff(T_) + (t >> 5) * 2 + 1] : 127u);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (r0 + i < a.rows) put2(out + (size_t)i * HD, y[i], false, sc[i]);
}
// rows r0, r0 + STEP, ...: all of them are requested before the first is stored
template <class T, int HD, int N, int STEP> __device__ __forceinline__ void read_keys(const C8ReadArgs& a, long r0, int u, int h) {
  using L = C8<HD>;
  const int T_ = 1 << a.c.psh;
  int slot[N];
  u32x2 c[N];
  float sc[N];
#pragma unroll
  for (int i = 0; i < N; ++i) slot[i] = a.slots[min(r0 + i * STEP, (long)a.rows - 1)];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const bool ok = slot[i] >= 0 && slot[i] < (long)a.c.n_pages << a.c.psh;
    const int s = ok ? slot[i] : 0, t = s & (T_ - 1);
    const uint8_t* page = a.c.data + ((size_t)(s >> a.c.psh) * a.c.hkv + h) * L::page_bytes(T_);
    c[i] = *(const u32x2*)(page + (size_t)t * HD + u * 8);
    const unsigned eb = page[L::soff(T_) + (t >> 5) * 2];
    if (!ok) c[i] = u32x2{0, 0};
    sc[i] = scale_of(ok ? eb : 127u);
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const long r = r0 + i * STEP;
    if (r >= a.rows) break;
    T* out = (T*)a.Ko + ((size_t)h * a.rows + r) * HD + u * 8;
    if constexpr (sizeof(T) == 2) {
      u32x4 y;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        y[2 * j] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c[i][j], sc[i], false));
        y[2 * j + 1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c[i][j], sc[i], true));
      }
      *(u32x4*)out = y;
    } else {
      float y[8];
      unpack4(y, c[i][0], sc[i]);
      unpack4(y + 4, c[i][1], sc[i]);
      *(f32x4*)out = f32x4{y[0], y[1], y[2], y[3]};
      *(f32x4*)(out + 4) = f32x4{y[4], y[5], y[6], y[7]};
    }
  }
}
constexpr int READ_ROWS = 64;      // rows of a workgroup
template <class T, int HD>
__global__ __launch_bounds__(NT) void cache8_read_kernel(C8ReadArgs a) {
  constexpr int U = HD / 8, W = NT / 64, V = 8 * 128 / HD;      // rows of a wave (values)
  const long r0 = (long)blockIdx.x * READ_ROWS;
  const int h = blockIdx.y;
  if (blockIdx.z == 0) {
    read_keys<T, HD, READ_ROWS * U / NT, NT / U>(a, r0 + threadIdx.x / U, threadIdx.x % U, h);
  } else {
#pragma unroll
    for (int i = 0; i < READ_ROWS; i += V * W) read_values<T, HD>(a, r0 + i + (threadIdx.x >> 6) * V, h);
  }
}

template <class T, int HD>
void write_t(const C8WriteArgs& a, hipStream_t st) {
  // a sequence of n rows touches at most (n + 2 U - 2) / U units of U, and no more than n
  auto units = [&](int u) { return (unsigned)std::min((long)a.rows, a.rows / u + 2L * a.batch); };
  const unsigned heads = (unsigned)a.c.hkv;
  const bool transposed = a.v_dim != 1;
  cache8_write_kernel<T, HD><<<dim3(units(UNIT), heads, transposed ? 1 : 2), NT, 0, st>>>(a);
  if (transposed) cache8_write_long_kernel<T, HD><<<dim3(units(LONG_UNIT), heads), LONG_UNIT * 4, 0, st>>>(a);
}

template <class T, int HD>
void read_t(const C8ReadArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)((a.rows + READ_ROWS - 1L) / READ_ROWS), (unsigned)a.c.hkv, 2);
  cache8_read_kernel<T, HD><<<grid, NT, 0, st>>>(a);
}

}  // namespace

void launch_cache8_write(int fp32, int hd, const C8WriteArgs& a, hipStream_t st) {
  if (fp32) hd == 128 ? write_t<float, 128>(a, st) : write_t<float, 64>(a, st);
  else hd == 128 ? write_t<f16, 128>(a, st) : write_t<f16, 64>(a, st);
}

void launch_cache8_read(int fp32, int hd, const C8ReadArgs& a, hipStream_t st) {
  if (fp32) hd == 128 ? read_t<float, 128>(a, st) : read_t<float, 64>(a, st);
  else hd == 128 ? read_t<f16, 128>(a, st) : read_t<f16, 64>(a, st);
}
