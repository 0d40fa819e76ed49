// Attention over the 8-bit paged prompt cache (layout: cache8.h): the kernels of
// attention_paged.h on e4m3 codes with a scale per 32 tokens and head.
//
// What bounds it: with few queries the cache's bytes, 2 D + 1/16 per key and head, at the
// 5.3 TB/s that a read of a large array reaches; with many the matrix instructions
// (4 D operations per key and query).
//
// A step's 32 keys are a block, so one scale goes into the expansion of all its keys, and one
// of its values.  Column kernel, 128 dimensions: 8 KB a step, 32 registers of a lane.
//   A key's fragments  two 16-byte pieces of its row, expanded two elements at a time
//   A value's          the two dimensions of a 16-byte piece, 8 keys each, likewise
// Row kernel: each of 512 threads expands 16 bytes of a tile's keys and 16 of its values,
// and scores are fp16 products like those of the fresh keys.
#include "attention_paged.h"
#include "cache8.h"

namespace {

// 8 codes, the element index rising with the byte
__device__ __forceinline__ void expand8(Frag<f16>& f, unsigned lo, unsigned hi, float sc) {
  const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, sc, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, sc, true);
  const f16x2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, sc, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, sc, true);
  f.v = f16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
__device__ __forceinline__ void expand8(Frag<float>& f, unsigned lo, unsigned hi, float sc) {
  const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(lo, sc, false), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(lo, sc, true);
  const f32x2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(hi, sc, false), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(hi, sc, true);
  f.v[0] = a[0]; f.v[1] = a[1]; f.v[2] = b[0]; f.v[3] = b[1]; f.v[4] = c[0]; f.v[5] = c[1]; f.v[6] = d[0]; f.v[7] = d[1];
}

__device__ __forceinline__ float scale_of(unsigned eb) { return __uint_as_float(eb << 23); }

// a piece's codes of the first m of its 8 keys; zeros after them, for a code there may be a NaN
// (a block without any key may never have been stored: its scale is taken as 1, for zeros times an infinite one are NaNs)
__device__ __forceinline__ u32x4 first_keys(u32x4 v, int m) {
  const unsigned lo = m >= 4 ? ~0u : m <= 0 ? 0u : (1u << (8 * m)) - 1;
  const unsigned hi = m >= 8 ? ~0u : m <= 4 ? 0u : (1u << (8 * m - 32)) - 1;
  return u32x4{v[0] & lo, v[1] & hi, v[2] & lo, v[3] & hi};
}

template <int HD> struct Fmt8 {
  using L = C8<HD>;
  static_assert(C8_BLOCK == STEP, "a step has one scale");
  __device__ static size_t page_bytes(int T) { return L::page_bytes(T); }
  // 16 bytes of a key: its fragments 2 i and 2 i + 1
  __device__ static constexpr int dim(int lg, int s) { return 64 * (s >> 1) + 16 * lg + 8 * (s & 1); }

  struct Raw {
    u32x4 k[2][HD / 64];      // the lane's dimensions of its two keys
    u32x4 v[HD / 32];         // its dimensions of its 8 keys, two at a time
    unsigned ks, vs;          // scale bytes
  };
  struct Lane {
    int koff, voff, soff;
    __device__ __forceinline__ Lane(int lg, int lc, int Tp)
        : koff(key_row(0, lc) * HD + lg * 16), voff(L::voff(Tp) + lg * L::VBLK + lc * 16), soff(L::soff(Tp)) {}
  };
  // of the step at position kp of the page p
  __device__ __forceinline__ static void load_keys(Raw& raw, const Lane& at, const uint8_t* p, int kp) {
    const uint8_t* kr = p + kp * HD + at.koff;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int i = 0; i < HD / 64; ++i) raw.k[kb][i] = *(const u32x4*)(kr + 4 * kb * HD + 64 * i);
    raw.ks = p[at.soff + (kp >> 5) * 2];
  }
  __device__ __forceinline__ static void load_values(Raw& raw, const Lane& at, const uint8_t* p, int kp) {
    const uint8_t* vr = p + kp * HD + at.voff;       // (kp / 8 blocks of 8 HD bytes)
#pragma unroll
    for (int i = 0; i < HD / 32; ++i) raw.v[i] = *(const u32x4*)(vr + 256 * i);
    raw.vs = p[at.soff + (kp >> 5) * 2 + 1];
  }
  template <class T, class S> __device__ __forceinline__ static void keys(const Raw& raw, int, S&& score) {
    const float sc = scale_of(raw.ks);
#pragma unroll
    for (int i = 0; i < HD / 32; ++i) {
      Frag<T> k[2];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) expand8(k[kb], raw.k[kb][i >> 1][2 * (i & 1)], raw.k[kb][i >> 1][2 * (i & 1) + 1], sc);
      score(k, i);
    }
  }
  template <class T, class V> __device__ __forceinline__ static void values(Raw& raw, int valid, int lg, V&& value) {
    const float sc = scale_of(valid > 0 ? raw.vs : 127u);
    if (valid < STEP) {
      const int m = valid - 8 * local_value(lg);
#pragma unroll
      for (int i = 0; i < HD / 32; ++i) raw.v[i] = first_keys(raw.v[i], m);
    }
#pragma unroll
    for (int i = 0; i < HD / 32; ++i) {
      Frag<T> a, b;
      expand8(a, raw.v[i][0], raw.v[i][1], sc);
      expand8(b, raw.v[i][2], raw.v[i][3], sc);
      value(a, 2 * i);
      value(b, 2 * i + 1);
    }
  }

  // Row kernel (128 dimensions).  Wave w expands a quarter of a tile's key block w / 2 (its
  // piece w % 2) and of the values of half w / 4 (piece w % 4), each lane the piece
  // whose fragments it reads itself.
  struct Row {
    using Stage = FreshStage;
    struct Query {};
    static constexpr int KROW = HD, KF = HD / 32, VF = HD / 16;
    static_assert(L::VBLK == 8 * KROW, "keys and values advance alike");
    struct Raw {
      u32x4 k, v;
      unsigned sc;            // both scale bytes of the half
    };
    int w, lane, vhalf, khalf;
    unsigned koff, voff, soff;
    __device__ __forceinline__ Row(int w, int lane, int Tp)
        : w(w), lane(lane), vhalf(w >> 2), khalf(w >> 2),
          koff((unsigned)(key_row((w >> 1) & 1, lane & 15) * KROW + (lane >> 4) * 16 + (w & 1) * 64)),
          voff((unsigned)(L::voff(Tp) + (lane >> 4) * L::VBLK + (w & 3) * 256 + (lane & 15) * 16)), soff((unsigned)L::soff(Tp)) {}
    // of the half whose codes begin at q, position kv of its page
    __device__ __forceinline__ void load(Raw& r, gbytes q, gbytes, int kv, int) const {
      r.k = *(gvec4)(q + local_value(koff));
      r.v = *(gvec4)(q + local_value(voff));
      r.sc = *(const __attribute__((address_space(1))) uint16_t*)(q + (soff + (kv >> 5) * 2 - kv * KROW));
    }
    __device__ __forceinline__ void fill(Stage& s, const Raw& r, int val) const {
      const int valid = (val >> (16 * vhalf)) & 0xffff;
      u32x4 v = r.v;
      if (valid < 32) v = first_keys(v, valid - 8 * local_value(lane >> 4));
      const float ks = scale_of(r.sc & 255u), vs = scale_of(valid > 0 ? r.sc >> 8 : 127u);
      Frag<f16> a, b, c, d;
      expand8(a, r.k[0], r.k[1], ks);
      expand8(b, r.k[2], r.k[3], ks);
      expand8(c, v[0], v[1], vs);
      expand8(d, v[2], v[3], vs);
      u32x4* kd = s.k + (((w >> 1) * KF + 2 * (w & 1)) * 64 + lane);
      kd[0] = __builtin_bit_cast(u32x4, a.v);
      kd[64] = __builtin_bit_cast(u32x4, b.v);
      u32x4* vd = s.v + ((vhalf * VF + 2 * (w & 3)) * 64 + lane);
      vd[0] = __builtin_bit_cast(u32x4, c.v);
      vd[64] = __builtin_bit_cast(u32x4, d.v);
    }
    __device__ __forceinline__ static Query query(const Frag<f16>*, float) { return Query{}; }
    template <int CB>
    __device__ __forceinline__ static void score(f32x4 (&sc)[CB][4], const f32x4 (&ref)[CB], const Stage& s, int lane,
                                                 const Query (&)[CB], const Frag<f16> (&q)[CB][4], float scale_log2) {
      score_halves<CB>(sc, ref, s, lane, q, scale_log2);
    }
  };
};

// Which kernel a call takes, by its number of columns (us on a GPU of 256 CUs, cached +
// fresh keys, heads of 128 dimensions, unless said otherwise):
//   COL1: up to 16 columns of a key head, a block to a workgroup.
//   COL2: more of them.  Against one block, it expands a step for 32 columns: B 32, 2000 + 8
//     keys, 8 rows, 28/4 heads: 25.2, one block 27.9.
//   WIDE: columns enough that the row kernel's workgroups of 256 occupy half of the CUs:
//       B 16, 1344 + 256 keys, 256 rows, 32/32 heads   125   COL2 206
//       B 16, 1000 + 128,      128,      16/16          35         39
//       B  8, 1000 + 128,      128,      32/32          38         43
//       B  4, 512 + 256,       256,      32/32          32         38
//       B  4, 1000 + 192,      192,      32/32          43         35    (so not here)
//       B  2, 4096 + 256,      256,      32/32         120         57    (nor here)
//       B  8, 1000 + 96,       96,       32/32          35         32    (nor here)
//     With 64 dimensions always two blocks of columns.  Four to a wave, each with its own, are faster only where
//     they make two workgroups for every CU: 256 rows, 32/32 heads, B 16, 1344 + 256 keys 90, four 77; B 8,
//     4096 + 256 107, four 132; B 8, 1344 + 256 51, four 56; 128 rows, B 16, 1000 + 128 40, four 54.
enum class Kind { COL1, COL2, WIDE };
Kind kind_of(int fp32, int batch, int G, int hq, int hkv, int hd) {
  const long ncol = (long)G * (hq / hkv), all = ncol * batch * hkv;
  // fp32: the matrix instructions take most of the time whatever the columns
  // share, and two blocks of accumulators do not fit the registers
  if (fp32 || ncol <= 16) return Kind::COL1;
  // at least half of the 256 columns of the workgroups in use
  const bool full = (ncol + 31) / 32 >= 4 * ((ncol + 255) / 256);
  return hd == 128 && full && all >= 1 << 15 ? Kind::WIDE : Kind::COL2;
}

template <class T, int HD>
void launch_kind(PagedAttnArgs a, hipStream_t st) {
  const Kind kind = kind_of(sizeof(T) == 4, a.batch, a.G, a.hq, a.hkv, a.hd);
  const long ncol = (long)a.G * (a.hq / a.hkv), cols = kind == Kind::COL1 ? 16 : kind == Kind::COL2 ? 32 : 256;
  const dim3 grid((unsigned)(a.hkv * ((ncol + cols - 1) / cols)), (unsigned)a.slots);
  // More workgroups than CUs: the longest sequences first, or the last ones to start are waited
  // for (16 sequences of 681 to 1971 cached and 256 fresh keys, 32 heads: 125 us, not 140).  In the
  // column kernel, several to a CU and shorter, it gives nothing (64 of 512 + 32 keys, 32 rows, 32 heads: 73 us, 72).
  a.sorted = kind == Kind::WIDE && a.batch > 1 && (long)grid.x * a.batch > 256;
  if (kind == Kind::COL1) {
    paged_columns_kernel<Fmt8<HD>, T, HD, 1, NWAVE><<<grid, 64 * NWAVE, 0, st>>>(a);
  } else if constexpr (sizeof(T) == 2) {
    if constexpr (HD == 128) {
      if (kind == Kind::WIDE) paged_rows_kernel<Fmt8<HD>><<<grid, 64 * RW, 0, st>>>(a);
      else paged_columns_kernel<Fmt8<HD>, T, HD, 2, NWAVE><<<grid, 64 * NWAVE, 0, st>>>(a);
    } else {
      paged_columns_kernel<Fmt8<HD>, T, HD, 2, NWAVE><<<grid, 64 * NWAVE, 0, st>>>(a);
    }
  }
  if (a.slots > a.batch) {
    constexpr int SL = 256 / (HD / 4);
    const long rows = (long)a.G * a.hq;
    if (rows < 1024) paged_merge_kernel<T, HD, SL><<<dim3((unsigned)rows, (unsigned)a.batch), 256, 0, st>>>(a);
    else paged_merge_kernel<T, HD, 1><<<dim3((unsigned)((rows + SL - 1) / SL), (unsigned)a.batch), 256, 0, st>>>(a);
  }
}

}  // namespace

// A workgroup of four waves takes 0.14 us for a step of its sequence (64 dimensions 0.09, fp32 0.61 and 0.33): expansion and
// matrix instructions fill its CU, and eight or sixteen waves take as long.  90 workgroups (123) reach what the memory
// gives, in fp32 it takes all of the CUs.  Cutting the sequences costs the merge's launch and a second pass over the
// queries, about 5 us.  So it has to save more steps than that is.  Unsplit and split, one row of 28/4 heads:
//                      128 dimensions   64           fp32
//   B  1,  1000 keys    8.5    9.7       6.5    9.1   24.1   13.9
//   B  1,  2000        12.9   10.0       9.6    9.3   43.4   14.1
//   B  4,  4000        21.8   10.5      15.8    9.7   81.9   14.7
//   B 16,  2000        13.6   13.0       9.8   11.1   43.4   20.3
//   B 16,  4000        22.8   18.0      16.1   13.6   82.4   32.4
//   B 32,  2000        14.5   20.6      10.4   14.3   43.5   34.0
// That is for sequences of one length, which is all that the host knows.  Where one of them may be
// far longer, its workgroup alone may walk for long, so a call of more than 1024 steps (140 us)
// is cut whatever the batch would take together; the chunks are made of the lengths there are, about
// one to a sequence where these are alike.  Up to 256 sequences: every wave scans their lengths.  Not where the
// key heads and blocks of one sequence are a round of workgroups by themselves (the partial results
// are twice its queries): there is nothing to gain.
//                                           unsplit   split
//   B 20, one of 131072 keys, 19 of 1000, 1 row, 32/8 heads     772    59
//   B 40, one of 131072, 39 of 1000,      1,     28/4           578    38
//   B 200, one of 40000, 199 of 1000,     1,     32/8           296   113
//   B 20, 33000 each,                     1,     28/4           217   128
//   B 20, 33000 each,                     1,     32/8           245   247
//   B 64, 33000 each,                     8,     28/4           575   588
//   B 64, 1000 each, max_cached 131072,   1,     32/8            24    28   (what a loose bound costs)
AttnSplit attn8_split(int fp32, int batch, int G, int hq, int hkv, int hd, int max_cached, int fresh) {
  const Kind kind = kind_of(fp32, batch, G, hq, hkv, hd);
  if (kind == Kind::WIDE) return AttnSplit{0, 0, batch, TILE};
  const long ncol = (long)G * (hq / hkv), groups = hkv * (kind == Kind::COL1 ? (ncol + 15) / 16 : (ncol + 31) / 32);
  const long steps = ((long)max_cached + STEP - 1) / STEP + ((fresh ? G : 0) + STEP - 1) / STEP;
  AttnSplit s{0, 2 * NWAVE, batch, STEP};
  // As many workgroups as CUs, where that is a good many chunks to a sequence (B 16, 8000 keys, 1 row, 28/4 heads: 27 us, 29
  // with four to a CU; B 4, 70001 to 131072: 75.5, 80.8).  Else one round of what the CUs hold: cutting B sequences by one
  // length leaves up to B chunks more than that length divides out (the first of the table above: 71, 57).
  const long round = 256 * (fp32 ? 3 : 256 / groups >= 4L * batch ? 1 : kind == Kind::COL1 ? 4 : 2);
  long target = round / groups - batch;
  const bool far = steps > 1024 && batch <= 256 && groups < round;
  if (far) target = std::max(target, (long)batch);
  // (the kernels count a batch's steps in 32 bits)
  if ((target <= batch && !far) || steps * batch > INT_MAX) return s;
  const long chunk = std::max((steps * batch + target - 1) / target, (long)s.chunk_min);
  const long busy = fp32 ? 256 : hd == 128 ? 90 : 123, cost = fp32 ? (hd == 128 ? 8 : 18) : hd == 128 ? 32 : 55;
  if (far || steps - std::max(chunk, steps * batch * groups / busy) > cost) {
    s.target = (int)target;
    s.slots = (int)std::min(target + batch, batch * ((steps + s.chunk_min - 1) / s.chunk_min));
  }
  return s;
}

void launch_attn8(int fp32, const PagedAttnArgs& a, hipStream_t st) {
  if (fp32) a.hd == 128 ? launch_kind<float, 128>(a, st) : launch_kind<float, 64>(a, st);
  else a.hd == 128 ? launch_kind<f16, 128>(a, st) : launch_kind<f16, 64>(a, st);
}
