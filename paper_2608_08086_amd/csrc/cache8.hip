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
#include <algorithm>

#include "cache8.h"

namespace {

constexpr int NT = 256;
constexpr int UNIT = 2 * C8_BLOCK;          // tokens of a workgroup: 128 bytes of a transposed row in fp16

typedef short i16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// inclusive sum over the wave's lanes
__device__ __forceinline__ int wave_scan(int x) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int t = __shfl_up(x, o, 64);
    if (lane >= o) x += t;
  }
  return x;
}

// The 64-token units of the batch, in sequence order: unit `key` is unit `first` + n of sequence b.
struct Span {
  int b, start, row0, row1, unit;   // rows row0 .. row1 - 1 at positions start ..; unit: number of the 64 tokens
};
__device__ __forceinline__ Span find_unit(const C8WriteArgs& a, int key) {
  const int lane = threadIdx.x & 63;
  int base = 0;
  for (int b0 = 0; b0 < a.batch; b0 += 64) {
    const int b = min(b0 + lane, a.batch - 1);
    // rows outside the arrays are none: neither is a sequence that does not fit the table
    const int s = a.start[b], r0 = min(max(a.row_off[b], 0), a.rows), r1 = min(max(a.row_off[b + 1], r0), a.rows);
    const long long cap = (long long)a.width << a.c.psh;
    const int fit = s < 0 ? 0 : (int)min((long long)(r1 - r0), max(cap - s, 0LL));
    const int n = b0 + lane < a.batch && fit > 0 ? (int)(((long long)s + fit - 1) / UNIT) - s / UNIT + 1 : 0;
    const int incl = wave_scan(n);
    const unsigned long long m = __ballot(base + incl > key);
    if (m) {
      const int at = __ffsll(m) - 1;
      Span v;
      v.b = b0 + at;
      v.start = __builtin_amdgcn_readlane(s, at);
      v.row0 = __builtin_amdgcn_readlane(r0, at);
      v.row1 = v.row0 + __builtin_amdgcn_readlane(fit, at);
      v.unit = v.start / UNIT + key - (base + __builtin_amdgcn_readlane(incl - n, at));
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

// A workgroup's two blocks.  TRANS: a head's values lie with their rows one element apart.
//   keys          thread: row tid / 8 of each block, HD / 8 dimensions from (tid % 8) HD / 8
//   values        wave w: 8-token block w of each block; lane (of HD / 2): dimensions 2 lane, 2 lane + 1
//   transposed    the same shares; lane l of wave w has 8-token block l % 4, so that the four
//                 lanes of a dimension read 64 consecutive bytes
template <class T, int HD, int KIND>     // 0 keys, 1 values, 2 values transposed
__device__ __forceinline__ void write_unit(const C8WriteArgs& a, const Span& v, int h) {
  using L = C8<HD>;
  constexpr int E = HD / 8, NB = UNIT / C8_BLOCK;       // elements of a thread of a block (values: 16, of fewer threads)
  constexpr int EV = KIND == 0 ? E : 16;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, Tp = 1 << a.c.psh;
  const T* src = KIND == 0 ? (const T*)a.K + h * a.k_head : (const T*)a.V + h * a.v_head;
  const bool on = KIND == 0 || HD == 128 || (KIND == 1 ? lane < HD / 2 : w < 2);
  // a thread's 8-token block and first dimension of its pair (values)
  const int tb = KIND == 1 ? w : lane & 3, pair = KIND == 1 ? lane : (lane >> 2) + 16 * w;
  const int dim = KIND == 0 ? (tid & 7) * E : 2 * min(pair, HD / 2 - 1);
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
    } else if constexpr (KIND == 1) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        T y[2];
        load_n<2>(y, src + row(8 * tb + i) * a.v_row + dim);
        t[k][i] = y[0];
        t[k][8 + i] = y[1];
      }
    } else {
      const int q = p0 + 8 * tb - v.start;
      if (q >= 0 && q + 8 <= n) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          T y[8];
          load_n<8>(y, src + (dim + s) * a.v_dim + v.row0 + q);
#pragma unroll
          for (int i = 0; i < 8; ++i) t[k][8 * s + i] = y[i];
        }
      } else {
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int i = 0; i < 8; ++i) t[k][8 * s + i] = src[(dim + s) * a.v_dim + row(8 * tb + i)];
      }
    }
  }
  // token of element e of this thread
  auto token = [&](int e) __attribute__((always_inline)) { return KIND == 0 ? tid >> 3 : 8 * tb + (e & 7); };
  const int off = KIND == 0 ? (tid >> 3) * HD + dim
                            : L::voff(Tp) + tb * L::VBLK + (dim % (HD / 16)) / 2 * 256 + dim / (HD / 16) * 16;
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
    uint8_t* scale = page[k] + L::soff(Tp) + (at[k] >> 5) * 2 + (KIND != 0);
    uint8_t* dst = page[k] + (size_t)at[k] * HD + off;      // (values: 32 tokens are 4 VBLK = 32 HD bytes as well)
    unsigned eb = exponent_of(m);
    if (p0 < v.start) {                   // joined: its earlier tokens, with their scale
      old[k] = min(max((unsigned)*scale, (unsigned)C8_EMIN), (unsigned)C8_EMAX);
      eb = max(eb, old[k]);
      unsigned c[EV / 4];
      if (on) __builtin_memcpy(c, __builtin_assume_aligned(dst, EV), EV);
#pragma unroll
      for (int e = 0; e < EV; e += 4) {
        float y[4];
        unpack4(y, on ? c[e / 4] : 0u, scale_of(old[k]));
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (p0 + token(e + i) < v.start) x[k][e + i] = y[i];
      }
      __syncthreads();                    // (uniform) the scale is read before it is written
    }
    if (eb == (unsigned)C8_EMAX) {        // only here can an element lie beyond 448
      const float most = 448.f * scale_of(eb);
#pragma unroll
      for (int e = 0; e < EV; ++e) x[k][e] = x[k][e] > most ? most : x[k][e] < -most ? -most : x[k][e];
    }
    unsigned c[EV / 4];
#pragma unroll
    for (int e = 0; e < EV; e += 4) c[e / 4] = pack4(&x[k][e], scale_of(eb));
    if (on) __builtin_memcpy(__builtin_assume_aligned(dst, EV), c, EV);
    if (tid == 0) *scale = (uint8_t)eb;
  }
}

template <class T, int HD, bool VT>
__global__ __launch_bounds__(NT) void cache8_write_kernel(C8WriteArgs a) {
  const Span v = find_unit(a, blockIdx.x);
  if (v.b < 0) return;
  if (blockIdx.z == 0) write_unit<T, HD, 0>(a, v, blockIdx.y);
  else write_unit<T, HD, VT ? 2 : 1>(a, v, blockIdx.y);
}

// Read back: a thread 8 dimensions of a row.  A slot outside the cache gives zeros.
template <class T, int HD>
__global__ __launch_bounds__(NT) void cache8_read_kernel(C8ReadArgs a) {
  constexpr int U = HD / 8, VF = HD / 16;
  using L = C8<HD>;
  const int u = threadIdx.x % U, h = blockIdx.y, T_ = 1 << a.c.psh;
  const long r = (long)blockIdx.x * (NT / U) + threadIdx.x / U;
  if (r >= a.rows) return;
  const bool value = blockIdx.z != 0;
  const int slot = a.slots[r];
  const bool ok = slot >= 0 && slot < (long)a.c.n_pages << a.c.psh;
  const int s = ok ? slot : 0, t = s & (T_ - 1);
  const uint8_t* page = a.c.data + ((size_t)(s >> a.c.psh) * a.c.hkv + h) * L::page_bytes(T_);
  unsigned c[2] = {0, 0};
  if (!value) {
    const u32x2 k = *(const u32x2*)(page + (size_t)t * HD + u * 8);
    c[0] = k[0];
    c[1] = k[1];
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int d = u * 8 + e;
      c[e >> 2] |= (unsigned)page[L::voff(T_) + (t >> 3) * L::VBLK + d % VF / 2 * 256 + d / VF * 16 + d % 2 * 8 + (t & 7)] << (8 * (e & 3));
    }
  }
  const unsigned eb = page[L::soff(T_) + (t >> 5) * 2 + value];
  if (!ok) c[0] = c[1] = 0;
  const float sc = scale_of(ok ? eb : 127u);
  T* out = (T*)(value ? a.Vo : a.Ko) + ((size_t)h * a.rows + r) * HD + u * 8;
  if constexpr (sizeof(T) == 2) {
    u32x4 y;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      y[2 * i] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c[i], sc, false));
      y[2 * i + 1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c[i], sc, true));
    }
    *(u32x4*)out = y;
  } else {
    float y[8];
    unpack4(y, c[0], sc);
    unpack4(y + 4, c[1], sc);
    *(f32x4*)out = f32x4{y[0], y[1], y[2], y[3]};
    *(f32x4*)(out + 4) = f32x4{y[4], y[5], y[6], y[7]};
  }
}

template <class T, int HD>
void write_t(const C8WriteArgs& a, hipStream_t st) {
  // a sequence of n rows touches at most (n + 126) / 64 units, and no more than n
  const long units = std::min((long)a.rows, a.rows / UNIT + 2L * a.batch);
  const dim3 grid((unsigned)units, (unsigned)a.c.hkv, 2);
  if (a.v_dim == 1) cache8_write_kernel<T, HD, false><<<grid, NT, 0, st>>>(a);
  else cache8_write_kernel<T, HD, true><<<grid, NT, 0, st>>>(a);
}

template <class T, int HD>
void read_t(const C8ReadArgs& a, hipStream_t st) {
  constexpr int per = NT / (HD / 8);
  const dim3 grid((unsigned)((a.rows + (long)per - 1) / per), (unsigned)a.c.hkv, 2);
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
