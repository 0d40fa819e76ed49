// Attention over the 4-bit paged prompt cache (layout: cache4.h): the kernels of
// attention_paged.h on e2m1 codes with a scale per 32 dimensions.
//
// What bounds it: with few queries the cache's bytes, 17/16 D per key and head, at the
// 5.3 TB/s that a read of a large array reaches; with many the matrix instructions of the
// softmax's fp16 probabilities and values (4 D operations per key and query in all).
//
// Column kernel: a step's 32 keys are 4352 bytes of a head of 128 dimensions, 20 registers of a lane.
// Measured, 128 dimensions, 32/8 heads, one row: 64 sequences of 4096 keys 53.8 us, 5.3 TB/s
// of stored bytes; one of 131072 keys (143 MB, 27 us at that rate) 29.4 us and 5.8 for the join.
//   A key's fragments  a lane's D/4 dimensions from lg D/4, which is a dwordx4 (D = 128) of the
//                 key's row, expanded two at a time.
//   A value's     a value unit, two of which elements one conversion makes (two dimensions of one
//                 key) and two byte permutes transpose (one dimension of two keys).
// Scores on the stored codes (as in the row kernel) cost more here than the expansion that they
// save: 8 sequences of 2000 + 8 keys, 8 rows, 28/4 heads 18.1 us, not 17.0.
#include "attention_paged.h"
#include "cache4.h"

namespace {

// scale byte i of w as the fp32 2^(byte - 127)
__device__ __forceinline__ float scale_of(unsigned w, int i) { return __uint_as_float(((w >> (8 * i)) & 255u) << 23); }

// the 8 codes of w times one scale
__device__ __forceinline__ void frag_codes(Frag<f16>& f, unsigned w, float sc) {
  const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, sc, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, sc, 1);
  const f16x2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, sc, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, sc, 3);
  f.v = f16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
__device__ __forceinline__ void frag_codes(Frag<float>& f, unsigned w, float sc) {
  const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, sc, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, sc, 1);
  const f32x2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, sc, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, sc, 3);
  f.v[0] = a[0]; f.v[1] = a[1]; f.v[2] = b[0]; f.v[3] = b[1]; f.v[4] = c[0]; f.v[5] = c[1]; f.v[6] = d[0]; f.v[7] = d[1];
}
// Dimensions 2 BYTE, 2 BYTE + 1 of 8 keys, key i's codes in byte BYTE0 + BYTE
// of word w[i * STRIDE / 4]: one fragment per dimension.
template <int B0, int B1>
__device__ __forceinline__ void frag_pair(Frag<f16>& lo, Frag<f16>& hi, const unsigned* w, int stride, const float* sc) {
  u32x4 l, h;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const unsigned a = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w[(2 * i) * stride / 2], sc[2 * i], B0));
    const unsigned b = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w[(2 * i + 1) * stride / 2], sc[2 * i + 1], B1));
    l[i] = __builtin_amdgcn_perm(b, a, 0x05040100u);
    h[i] = __builtin_amdgcn_perm(b, a, 0x07060302u);
  }
  lo.v = __builtin_bit_cast(f16x8, l);
  hi.v = __builtin_bit_cast(f16x8, h);
}
template <int B0, int B1>
__device__ __forceinline__ void frag_pair(Frag<float>& lo, Frag<float>& hi, const unsigned* w, int stride, const float* sc) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[(2 * i) * stride / 2], sc[2 * i], B0);
    const f32x2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[(2 * i + 1) * stride / 2], sc[2 * i + 1], B1);
    lo.v[2 * i] = a[0]; hi.v[2 * i] = a[1];
    lo.v[2 * i + 1] = b[0]; hi.v[2 * i + 1] = b[1];
  }
}

// The value fragments of dimensions lc D/16 + 2 P and + 2 P + 1 of a unit, 8 keys each.
template <class T, int HD, int P>
__device__ __forceinline__ void value_pair(Frag<T>& lo, Frag<T>& hi, const unsigned* w, const float* sc) {
  if constexpr (HD == 128) frag_pair<P, P>(lo, hi, w, 2, sc);      // one dword a key
  else frag_pair<P, P + 2>(lo, hi, w, 1, sc);                      // two keys a dword
}

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef unsigned u32x6 __attribute__((ext_vector_type(6)));
typedef _Float16 f16x32 __attribute__((ext_vector_type(32)));
typedef float f32x32 __attribute__((ext_vector_type(32)));

// Four e2m3 terms of a lane's 32 query elements times `mul`, and their scale bytes.
struct QTerms {
  u32x6 t[4];
  unsigned scale;    // byte i: the biased exponent of term i
};
__device__ __forceinline__ QTerms query_terms(const Frag<f16>* q, float mul) {
  QTerms r;
  f32x32 x;
  // max |q| as an integer: infinities and NaN above the rest
  typedef unsigned short u16x8 __attribute__((ext_vector_type(8)));
  u16x8 t = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) t = __builtin_elementwise_max(t, __builtin_bit_cast(u16x8, q[i].v) & (unsigned short)0x7fff);
  unsigned short th = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) th = max(th, t[e]);
  const unsigned top = __float_as_uint((float)__builtin_bit_cast(f16, th) * mul);
  // s1 = 2^(e1 - 127): the least power of two with max |q| <= 7.5 s1; 0 and tiny values take any
  const unsigned e1 = max((top + 0x0fffffu) >> 23, 80u) - 2u;
  const float unit = mul * __uint_as_float((254u - e1) << 23);      // q mul rounded to fp32, in units of s1
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) x[8 * i + e] = fmaf((float)q[i].v[e], unit, 0.f);
  // a residual of t1 is at most s1 / 4, of the others an eighth of their scale: at most 4 of the next
  // scale.  Through fp16 only to choose the nearest e2m3, in units of s1, where fp16's own steps
  // (2^-24 at least) are far below the fourth term's 2^-17; the residual is kept in fp32.
  constexpr unsigned below[4] = {0, 4, 9, 14};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float s = __uint_as_float((127u - below[i]) << 23);
    r.t[i] = __builtin_amdgcn_cvt_scalef32_pk32_fp6_f16(__builtin_convertvector(x, f16x32), s);
    x -= __builtin_amdgcn_cvt_scalef32_pk32_f32_fp6(r.t[i], s);
  }
  // an infinite or NaN query element: NaN scores
  r.scale = (top >= 0x7f800000u ? 255u : e1) | (e1 - 4u) << 8 | (e1 - 9u) << 16 | (e1 - 14u) << 24;
  return r;
}

__device__ __forceinline__ i32x8 operand6(const u32x6& t) {
  return i32x8{(int)t[0], (int)t[1], (int)t[2], (int)t[3], (int)t[4], (int)t[5], 0, 0};
}

// scores += codes (lane's 32, scale byte KB of ks) x term I
template <int KB, int I>
__device__ __forceinline__ f32x4 mfma_codes(const u32x4& k, unsigned ks, const QTerms& q, f32x4 c) {
  const i32x8 a = {(int)k[0], (int)k[1], (int)k[2], (int)k[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, operand6(q.t[I]), c, 4, 2, KB, (int)ks, I, (int)q.scale);
}

struct RowStage {
  u32x4 v[2 * 8 * 64];       // value fragments [half][j][lane]
  u32x4 k[4 * 64];           // codes [kb][lane]
  uint16_t ks[128];          // a lane's scales of the four key blocks
};
template <int HD> struct Fmt4 {
  using L = C4<HD>;
  __device__ static size_t page_bytes(int T) { return L::page_bytes(T); }
  __device__ static constexpr int dim(int lg, int s) { return lg * (HD / 4) + 8 * s; }

  // A step's stored bytes as a lane holds them.
  struct Raw {
    unsigned k[2][HD / 32];      // the lane's dimensions of its two keys
    unsigned v[L::VUNIT / 4];
    u32x2 ks, vs;                // scales of 8 keys each
  };

  // a lane's two keys' rows, its value unit, their scales
  struct Lane {
    int koff, voff, ksoff, vsoff;
    __device__ __forceinline__ Lane(int lg, int lc, int Tp)
        : koff(key_row(0, lc) * L::KROW + lg * (HD / 8)), voff(L::voff(Tp) + lg * L::VBLK + lc * L::VUNIT),
          ksoff(L::ksoff(Tp) + (lc >> 2) * L::SBLK + (lg * (HD / 4) / 32) * 8),
          vsoff(L::vsoff(Tp) + lg * L::SBLK + (lc * (HD / 16) / 32) * 8) {}
  };
  // of the step at position kp of the page p
  __device__ __forceinline__ static void load_keys(Raw& raw, const Lane& at, const uint8_t* p, int kp) {
    const uint8_t* kr = p + kp * L::KROW + at.koff;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) __builtin_memcpy(raw.k[kb], __builtin_assume_aligned(kr + 4 * kb * L::KROW, HD / 8), HD / 8);
    raw.ks = *(const u32x2*)(p + (kp >> 3) * L::SBLK + at.ksoff);
  }
  __device__ __forceinline__ static void load_values(Raw& raw, const Lane& at, const uint8_t* p, int kp) {
    __builtin_memcpy(raw.v, __builtin_assume_aligned(p + (kp >> 3) * L::VBLK + at.voff, 16), L::VUNIT);
    raw.vs = *(const u32x2*)(p + (kp >> 3) * L::SBLK + at.vsoff);
  }
  template <class T, class S> __device__ __forceinline__ static void keys(const Raw& raw, int lc, S&& score) {
    const float ks[2] = {scale_of(raw.ks[0], lc & 3), scale_of(raw.ks[1], lc & 3)};
#pragma unroll
    for (int i = 0; i < HD / 32; ++i) {
      Frag<T> k[2];
      frag_codes(k[0], raw.k[0][i], ks[0]);
      frag_codes(k[1], raw.k[1][i], ks[1]);
      score(k, i);
    }
  }
  template <class T, class V> __device__ __forceinline__ static void values(const Raw& raw, int valid, int lg, V&& value) {
    float vs[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) vs[i] = scale_of(raw.vs[i >> 2], i & 3);
    if (valid < STEP) {
      // keys past the end: scale 0, hence zeros, whatever is stored there
      const int m = valid - 8 * local_value(lg);
#pragma unroll
      for (int i = 0; i < 8; ++i) vs[i] = i < m ? vs[i] : 0.f;
    }
    auto pair = [&](auto p) __attribute__((always_inline)) {
      Frag<T> lo, hi;
      value_pair<T, HD, p.value>(lo, hi, raw.v, vs);
      value(lo, 2 * p.value);
      value(hi, 2 * p.value + 1);
    };
    pair(std::integral_constant<int, 0>());
    pair(std::integral_constant<int, 1>());
    if constexpr (HD == 128) {
      pair(std::integral_constant<int, 2>());
      pair(std::integral_constant<int, 3>());
    }
  }

  // Row kernel (128 dimensions): scores on the codes themselves.  The fp4 x fp6 MFMA (16x16x128, block scales) takes
  // a key's 32 codes of a lane and their scale byte as they are stored, at the
  // rate of an fp16 16x16x32, so four times its work.  A query is the sum of four
  // e2m3 terms per 32 dimensions, each term's scale a power of two:
  //   q = t1 + t2 + t3 + t4 + r,  |r| <= 2^-17 s1,  s1 = the scale of t1, max |q| > 3.75 s1,
  // an error of at most 2^-18.9 of the largest element of the 32, less than the fp32 sums may be
  // off by.  Four MFMAs do what four fp16 ones would, and no key is expanded.  (Three terms:
  // 2^-13.9, which is more than the fp16 probabilities' rounding where scores are large or one of the 32
  // elements outweighs the others; 39.2 us in place of 40.7 for 8 sequences of 512 + 256 keys, 174 in
  // place of 190 for 8 of 5376.)  The queries
  // carry the softmax's factor, and the MFMA starts from minus the column's reference,
  // so that a score comes out as the exponent of its probability.
  // Measured, 32/32 heads, 256 rows, back to back (the clock falls by a tenth in the longer ones): 8 sequences of
  // 5376 keys 190 to 200 us (0.95 to 0.90 PF/s; a large fp16 library product reaches 1.22 on this GPU),
  // 8 of 512 cached and 256 fresh keys 40 us, 16 of 1344 and 256 132 to 159.  Of the cycles the
  // matrix pipes are busy in 56 %, a wave waits in 21 %.  A tile takes about 3900 in both halves: P V 730,
  // scores 790, exponentials and loads 600 to 800, softmax 300, expansion 330, LDS stores 210 to
  // 340, and the rest waiting at the barriers, for the halves are not equally long.
  struct Row {
    using Stage = RowStage;
    using Query = QTerms;
    static constexpr int KROW = L::KROW, VF = HD / 16;
    static_assert(L::VBLK == 8 * L::KROW, "keys and values advance alike");
    // A thread's value unit (block vblk of the half that its wave has, unit u), of which it
    // expands byte vbyte of each key; and 16 bytes of codes (waves 0-3: key block w)
    // or of key scales (waves 4, 5: half w & 1; 6, 7 the same, unused).
    struct Raw {
      u32x4 v[2];
      u32x2 vs;
      u32x4 k;
    };
    int w, lane, vhalf, vblk, u, vbyte, khalf;
    unsigned voff, vsoff, koff;
    __device__ __forceinline__ Row(int w, int lane, int Tp)
        : w(w), lane(lane), vhalf(w & 1), vblk(lane >> 4), u(lane & 15), vbyte(w >> 1), khalf(w < 4 ? w >> 1 : w & 1),
          voff((unsigned)(L::voff(Tp) + vblk * L::VBLK + u * L::VUNIT)),
          vsoff((unsigned)(L::vsoff(Tp) + vblk * L::SBLK + (u >> 2) * 8)),
          koff(w < 4 ? (unsigned)(key_row(w & 1, u) * L::KROW + vblk * 16)
                     : (unsigned)(L::ksoff(Tp) + (u >> 2) * L::SBLK + vblk / 2 * 16)) {}
    // of the values' half (codes from q, position kv of its page) and the keys' (qk, kk)
    __device__ __forceinline__ void load(Raw& r, gbytes q, gbytes qk, int kv, int kk) const {
      constexpr int BACK = L::KROW - L::SBLK / 8;   // scales advance by so much less than codes
      const unsigned vo = local_value(voff), so = local_value(vsoff) - kv * BACK, ko = local_value(koff) - (w < 4 ? 0 : kk * BACK);
      r.v[0] = *(gvec4)(q + vo);
      r.v[1] = *(gvec4)(q + 16 + vo);
      r.vs = *(gvec2)(q + so);
      r.k = *(gvec4)(qk + ko);
    }
    __device__ __forceinline__ void fill(Stage& s, const Raw& r, int val) const {
      const int valid = (val >> (16 * vhalf)) & 0xffff;
      float sc[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) sc[i] = scale_of(r.vs[i >> 2], i & 3);
      if (valid < 32) {
        const int n = valid - 8 * local_value(vblk);
#pragma unroll
        for (int i = 0; i < 8; ++i) sc[i] = i < n ? sc[i] : 0.f;
      }
      unsigned x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = r.v[i >> 2][i & 3] >> (8 * vbyte);
      Frag<f16> lo, hi;
      value_pair<f16, HD, 0>(lo, hi, x, sc);
      u32x4* d = s.v + ((vhalf * VF + 2 * vbyte) * 64 + lane);
      d[0] = __builtin_bit_cast(u32x4, lo.v);
      d[64] = __builtin_bit_cast(u32x4, hi.v);
      const int lg = vblk, lc = u;
      if (w < 4) {
        s.k[w * 64 + lane] = r.k;
      } else if (w < 6) {
        // the lane's two keys of this half: bytes lc & 3 of both words of its 8
        const unsigned a0 = lg & 1 ? r.k[2] : r.k[0], a1 = lg & 1 ? r.k[3] : r.k[1];
        s.ks[2 * lane + khalf] = (uint16_t)__builtin_amdgcn_perm(a1, a0, 0x0c0c0400u + (unsigned)(lc & 3) * 0x0101u);
      }
    }
    __device__ __forceinline__ static Query query(const Frag<f16>* q, float scale_log2) { return query_terms(q, scale_log2); }
    template <int CB>
    __device__ __forceinline__ static void score(f32x4 (&sc)[CB][4], const f32x4 (&ref)[CB], const Stage& s, int lane,
                                                 const Query (&q)[CB], const Frag<f16> (&)[CB][4], float) {
      const unsigned ks = *(const unsigned*)&s.ks[2 * lane];
      u32x4 k[4];
#pragma unroll
      for (int kb = 0; kb < 4; ++kb) k[kb] = s.k[kb * 64 + lane];
      // the smallest term first; eight independent sums, one MFMA of each in turn
      auto term = [&](auto x) __attribute__((always_inline)) {
        constexpr int I = x.value;
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
          sc[cb][0] = mfma_codes<0, I>(k[0], ks, q[cb], I == 3 ? ref[cb] : sc[cb][0]);
          sc[cb][1] = mfma_codes<1, I>(k[1], ks, q[cb], I == 3 ? ref[cb] : sc[cb][1]);
          sc[cb][2] = mfma_codes<2, I>(k[2], ks, q[cb], I == 3 ? ref[cb] : sc[cb][2]);
          sc[cb][3] = mfma_codes<3, I>(k[3], ks, q[cb], I == 3 ? ref[cb] : sc[cb][3]);
        }
        __builtin_amdgcn_sched_barrier(0);
      };
      __builtin_amdgcn_sched_barrier(0);
      term(std::integral_constant<int, 3>());
      term(std::integral_constant<int, 2>());
      term(std::integral_constant<int, 1>());
      term(std::integral_constant<int, 0>());
    }
  };
};

// Which kernel a call takes, by its number of columns (us on a GPU of 256 CUs, cached +
// fresh keys, heads of 128 dimensions, unless said otherwise):
//   COL1: up to 16 columns of a key head, a block to a workgroup.
//   COL2: more of them.  Against one block, it expands a step for 32 columns; against four
//     (64), two waves fit a SIMD: B 32, 2000 + 8 keys, 8 rows, 28/4 heads: 18.5, four 28.4.
//   WIDE: columns enough that a workgroup's 256 (head_dim 128, row kernel) or 4 x 64
//     (head_dim 64, four blocks a wave) occupy half of the CUs, or all of them twice:
//       B 16, 1344 + 256 keys, 256 rows, 32/32 heads   153   COL2 208
//       B  8, 512 + 256,       256,      32/32          41         64
//       B 16, 1000 + 128,      128,      16/16          35         39
//       B  4, 512 + 256,       256,      32/32          34         34
//       B  2, 4096 + 256,      256,      32/32         117         54    (so not here)
//       B  8, 1024 + 70,        70,      32/32          32         29    (nor here)
//       B 16, 1344 + 256,      256,      32/32, 64 dim. 83         98
//       B  8, 512 + 256,       256,      16/16, 64 dim. 27         19    (nor here)
enum class Kind { COL1, COL2, WIDE };
Kind kind_of(int fp32, int batch, int G, int hq, int hkv, int hd) {
  const long ncol = (long)G * (hq / hkv), all = ncol * batch * hkv;
  // fp32: the matrix instructions take most of the time whatever the columns
  // share, and two blocks of accumulators do not fit the registers
  if (fp32 || ncol <= 16) return Kind::COL1;
  // at least half of the 256 columns of the workgroups in use
  const bool full = (ncol + 31) / 32 >= 4 * ((ncol + 255) / 256);
  return full && all >= (hd == 128 ? 1 << 15 : 1 << 16) ? Kind::WIDE : Kind::COL2;
}

template <class T, int HD>
void launch_kind(PagedAttnArgs a, hipStream_t st) {
  const Kind kind = kind_of(sizeof(T) == 4, a.batch, a.G, a.hq, a.hkv, a.hd);
  const long ncol = (long)a.G * (a.hq / a.hkv), cols = kind == Kind::COL1 ? 16 : kind == Kind::COL2 ? 32 : 256;
  const dim3 grid((unsigned)(a.hkv * ((ncol + cols - 1) / cols)), (unsigned)a.slots);
  // More workgroups than CUs: the longest sequences first, or the last ones to start are waited
  // for (16 sequences of 681 to 1971 cached and 256 fresh keys, 32 heads: 155 us, not 166).  In the
  // column kernel, several to a CU and shorter, it costs more than it gives (64 of 512 + 32
  // keys, 32 rows, 32 heads: 65 us, not 54).
  a.sorted = kind == Kind::WIDE && a.batch > 1 && (long)grid.x * a.batch > 256;
  if (kind == Kind::COL1) {
    paged_columns_kernel<Fmt4<HD>, T, HD, 1, NWAVE><<<grid, 64 * NWAVE, 0, st>>>(a);
  } else if constexpr (sizeof(T) == 2) {
    if (kind == Kind::COL2) paged_columns_kernel<Fmt4<HD>, T, HD, 2, NWAVE><<<grid, 64 * NWAVE, 0, st>>>(a);
    else if constexpr (HD == 128) paged_rows_kernel<Fmt4<HD>><<<grid, 64 * RW, 0, st>>>(a);
    else paged_columns_kernel<Fmt4<HD>, T, HD, 4, 1><<<grid, 64 * NWAVE, 0, st>>>(a);
  }
  if (a.slots > a.batch) {
    constexpr int SL = 256 / (HD / 4);
    const long rows = (long)a.G * a.hq;
    if (rows < 1024) paged_merge_kernel<T, HD, SL><<<dim3((unsigned)rows, (unsigned)a.batch), 256, 0, st>>>(a);
    else paged_merge_kernel<T, HD, 1><<<dim3((unsigned)((rows + SL - 1) / SL), (unsigned)a.batch), 256, 0, st>>>(a);
  }
}

}  // namespace

// A workgroup of four waves takes about 0.13 us for a step of its sequence, and about 160 of
// them together what the memory (one block) or the CUs (two) can do.  Cutting the sequences
// costs the merge's launch and a second pass over the queries, 4 to 8 us (part of it the merge's own
// scan of the lengths), so it has to save more than 56 steps.  Unsplit and split:
//   B  1,  2500 keys,  1 row, 32/8 heads    13.9   15.0
//   B  4,  2500,       1,     32/8          14.7   13.7
//   B  4,  4096,       1,     32/8          20.9   14.7
//   B 32,  2500,       1,     32/8          18.4   22.8
//   B  8,  2000 + 8,   8,     28/4          16.8   20.6
// That is for sequences of one length, which is all that the host knows.  Where one of them may be
// far longer, its workgroup alone may walk for long, so a call of more than 1024 steps (130 us)
// is cut whatever the batch would take together; the chunks are made of the lengths there are, about
// one to a sequence where these are alike.  Up to 256 sequences: every wave scans their lengths.  Not where the
// key heads and blocks of one sequence are a round of workgroups by themselves (the partial results
// are twice its queries): there is nothing to gain (fp32, 128 rows, 32/32 heads, half a round: 1048, 1025).
//                                           unsplit   split
//   B 20, one of 131072 keys, 19 of 1000, 1 row, 32/8 heads     737    37
//   B 40, one of 131072, 39 of 1000,      1,     28/4           550    27
//   B 200, one of 40000, 199 of 1000,     1,     32/8           244    76
//   B 20, 33000 each,                     1,     32/8           211   147
//   B 64, 33000 each,                     1,     32/8           379   388
//   B 64, 33000 each,                     8,     28/4           401   415
//   B 64, 1000 each, max_cached 131072,   1,     32/8            12    18   (what a loose bound costs)
//   B 200, 1000 each, max_cached 131072,  1,     32/8            28    52
AttnSplit attn4_split(int fp32, int batch, int G, int hq, int hkv, int hd, int max_cached, int fresh) {
  const Kind kind = kind_of(fp32, batch, G, hq, hkv, hd);
  if (kind == Kind::WIDE) return AttnSplit{0, 0, batch, hd == 128 ? TILE : STEP};
  const long ncol = (long)G * (hq / hkv), groups = hkv * (kind == Kind::COL1 ? (ncol + 15) / 16 : (ncol + 31) / 32);
  const long steps = ((long)max_cached + STEP - 1) / STEP + ((fresh ? G : 0) + STEP - 1) / STEP;
  AttnSplit s{0, 2 * NWAVE, batch, STEP};
  // One round of what the CUs hold (four workgroups of one block each, two of the others): cutting
  // B sequences by one length leaves up to B chunks more than that length divides out.
  const long round = 256 * (kind == Kind::COL1 && !fp32 ? 4 : 2);
  long target = round / groups - batch;
  const bool far = steps > 1024 && batch <= 256 && groups < round;
  if (far) target = std::max(target, (long)batch);
  // (the kernels count a batch's steps in 32 bits)
  if ((target <= batch && !far) || steps * batch > INT_MAX) return s;
  const long chunk = std::max((steps * batch + target - 1) / target, (long)s.chunk_min);
  if (far || steps - std::max(chunk, steps * batch * groups / 160) > 56) {
    s.target = (int)target;
    s.slots = (int)std::min(target + batch, batch * ((steps + s.chunk_min - 1) / s.chunk_min));
  }
  return s;
}

void launch_attn4(int fp32, const PagedAttnArgs& a, hipStream_t st) {
  if (fp32) a.hd == 128 ? launch_kind<float, 128>(a, st) : launch_kind<float, 64>(a, st);
  else a.hd == 128 ? launch_kind<f16, 128>(a, st) : launch_kind<f16, 64>(a, st);
}
