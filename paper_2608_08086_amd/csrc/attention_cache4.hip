// Non-causal attention over the 4-bit paged prompt cache and an optional
// fresh segment (layout: cache4.h):
//   O = softmax([q K4^T, q K2^T] / sqrt(D)) [V4; V2]
// per sequence, no mask other than key validity.  Stored elements are exact in
// fp16, so for fp16 queries the column kernel's only roundings are those of the fp16
// attention beside it: the probabilities to fp16 and the output to bf16 (scores, running
// maximum and sum and the accumulators are fp32).  The row kernel also writes a query as
// four short terms; see there.
//
// What bounds it: with few queries the cache's bytes, 17/16 D per key and head, at the
// 5.3 TB/s that a read of a large array reaches; with many the matrix instructions of the
// softmax's fp16 probabilities and values (4 D operations per key and query in all).
//
// Column kernel: the queries that share a key head are the columns of the
// score MFMA (G rows of hq / hkv heads, 16 CB columns to a wave), and a
// wave expands what it multiplies: 32 keys at a time (4352 bytes of a head of 128
// dimensions, 20 registers of a lane), straight from memory to the operands,
// the next ones requested before these are used.  The workgroup's four waves take turns
// along its share of the keys, and their partial softmaxes are joined in LDS (KW = 4); or
// each wave has columns of its own, and there is no barrier at all (KW = 1).
// Measured, 128 dimensions, 32/8 heads, one row: 64 sequences of 4096 keys 53.8 us, 5.3 TB/s
// of stored bytes; one of 131072 keys (143 MB, 27 us at that rate) 29.4 us and 5.8 for the join.
//
//   S^T = K Q^T   A operand: lane (lc, lg) holds key att key(lc) and the D/4
//                 dimensions from lg D/4, which is a dwordx4 (D = 128) of the
//                 key's row, expanded two at a time; any order of the
//                 dimensions will do as long as Q's fragments have the same.
//   O^T = V^T P^T A operand: lane (lc, lg) holds the D/16 dimensions from
//                 lc D/16 of the 8 keys 8 lg .. 8 lg + 7, a value unit, two of
//                 which elements one conversion makes (two dimensions of one
//                 key) and two byte permutes transpose (one dimension of two keys).
// The keys of a score block are ordered so that a lane's scores of the two
// blocks are the 8 keys that its P V operand needs.
// Scores on the stored codes (as in the row kernel) cost more here than the expansion that they
// save: 8 sequences of 2000 + 8 keys, 8 rows, 28/4 heads 18.1 us, not 17.0.
#include <algorithm>
#include <climits>

#include "cache4.h"

namespace {

constexpr int STEP = 32;          // keys of one step of the column kernel
constexpr int TILE = 64;          // keys of one step of the row kernel

__device__ __forceinline__ float max_groups(float x) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float sum_groups(float x) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// x, to be looked at only here: what is computed from it is not moved out of a
// loop, where it would hold a register for a rare branch (or, zero-extended, two)
__device__ __forceinline__ int local_value(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// scale byte i of w as the fp32 2^(byte - 127)
__device__ __forceinline__ float scale_of(unsigned w, int i) { return __uint_as_float(((w >> (8 * i)) & 255u) << 23); }

// Operand fragments: 8 elements of the contraction index per lane for fp16
// (16x16x32), one per lane and instruction for fp32 (16x16x4, eight of them).
template <class T> struct Frag;
template <> struct Frag<f16> { f16x8 v; };
template <> struct Frag<float> { float v[8]; };

__device__ __forceinline__ f32x4 mfma8(const Frag<f16>& a, const Frag<f16>& b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a.v, b.v, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma8(const Frag<float>& a, const Frag<float>& b, f32x4 c) {
#pragma unroll
  for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[e], b.v[e], c, 0, 0, 0);
  return c;
}

// 8 consecutive elements of a fragment from memory
__device__ __forceinline__ void frag_load(Frag<f16>& f, const f16* p) { f.v = __builtin_bit_cast(f16x8, *(const u32x4*)p); }
__device__ __forceinline__ void frag_load(Frag<float>& f, const float* p) {
  const f32x4 a = *(const f32x4*)p, b = *(const f32x4*)(p + 4);
#pragma unroll
  for (int e = 0; e < 4; ++e) { f.v[e] = a[e]; f.v[4 + e] = b[e]; }
}
template <class T> __device__ __forceinline__ void frag_zero(Frag<T>& f) {
#pragma unroll
  for (int e = 0; e < 8; ++e) f.v[e] = (T)0.f;
}
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

// key (of 32) of row r of score block kb
__device__ __forceinline__ int key_row(int kb, int r) { return 8 * (r >> 2) + 4 * kb + (r & 3); }

template <class T> struct OutOf { using type = bf16; };
template <> struct OutOf<float> { using type = float; };

// Running maximum before the first key: below every score, and finite, so that
// no difference of maxima is a NaN; and after keys whose scores are all -infinity
// (an infinite query or key element), so that a row of these is told from one without keys.
constexpr float M_NONE = -3.0e38f, M_KEYS = -2.9e38f;

// The softmax's sum, of running maximum m: without keys 0, with none but -infinite scores NaN.
__device__ __forceinline__ float final_sum(float l, float m) { return l == 0.f && m > M_NONE ? NAN : l; }

// four dimensions of an output row: x / l, or zeros where there was no key
template <class OT>
__device__ __forceinline__ void store_row4(OT* p, f32x4 x, float l) {
  const float inv = l == 0.f ? 0.f : 1.0f / l;
  if constexpr (sizeof(OT) == 2) {
    bf16x4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = (bf16)(x[e] * inv);
    *(bf16x4*)p = v;
  } else {
    *(f32x4*)p = x * inv;
  }
}

// Work of one call.  Sequence b's keys are steps of 32 (row kernel: tiles of 64; cached, then fresh
// ones).  The row kernel takes a sequence whole; the column kernel's sequences are cut into
// chunks of one length for the whole batch, so that a ragged batch fills the
// GPU evenly.  Chunk `slot` of the batch, in sequence order, is a workgroup's
// share for every key head and column block; the lengths are on the device, so
// each wave finds its chunk by a scan over the batch (64 sequences at a time,
// lane-parallel).  Sequences of one chunk are finished by their workgroup, the
// others by the merge.
struct SeqView {
  int len, nfresh, rows, steps1, steps;
};
__device__ __forceinline__ SeqView seq_view(const Attn4Args& a, int b) {
  SeqView v;
  const int cap = (int)min((long long)a.max_cached, (long long)a.width << a.c.psh);
  v.len = min(max(a.cached_len[b], 0), cap);
  v.rows = a.resp_len ? min(max(a.resp_len[b], 0), a.G) : a.G;
  v.nfresh = a.K2 ? v.rows : 0;
  v.steps1 = (int)(((unsigned)v.len + a.step - 1) / a.step);
  v.steps = v.steps1 + (v.nfresh + a.step - 1) / a.step;
  return v;
}

// inclusive sum over the wave's lanes
__device__ __forceinline__ int wave_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);    // row_shr 1, 2, 4, 8
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);   // row_bcast 15, 31
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
  return x;
}

struct Work {
  int b, first, nsplit, chunk;   // b < 0: no such chunk
};

// Sequence `key` in the order of falling length, of the 64 that it is one of.
__device__ __forceinline__ int by_length(const Attn4Args& a, int key) {
  const int lane = threadIdx.x & 63, b0 = key & ~63, n = min(a.batch - b0, 64);
  const int mine = seq_view(a, b0 + min(lane, n - 1)).steps;
  int rank = lane < n ? 0 : 64;
  for (int i = 0; i < n; ++i) {
    const int other = __builtin_amdgcn_readlane(mine, i);
    rank += (other > mine) | ((other == mine) & (i < lane));
  }
  return b0 + __ffsll(__ballot(rank == key - b0)) - 1;
}

// BY_SEQ: the chunks of sequence `key`; else the sequence of chunk `key`.
template <bool BY_SEQ>
__device__ __forceinline__ Work find_work(const Attn4Args& a, int key) {
  const int lane = threadIdx.x & 63;
  Work w{-1, 0, 1, INT_MAX};
  if (a.target == 0) {           // no splits: chunk b is sequence b
    w.b = key;
    w.first = key;
    return w;
  }
  long long total = 0;
  int mine = 0;                  // steps of sequence `lane` of the last 64
  for (int b0 = 0; b0 < a.batch; b0 += 64) {
    mine = b0 + lane < a.batch ? seq_view(a, b0 + lane).steps : 0;
    total += __builtin_amdgcn_readlane(wave_scan(mine), 63);
  }
  w.chunk = (int)max((total + a.target - 1) / a.target, (long long)a.chunk_min);
  int base = 0;
  for (int b0 = 0; b0 < a.batch; b0 += 64) {
    if (a.batch > 64) mine = b0 + lane < a.batch ? seq_view(a, b0 + lane).steps : 0;
    const int n = b0 + lane < a.batch ? max(1, (mine + w.chunk - 1) / w.chunk) : 0;
    const int incl = wave_scan(n), sum = __builtin_amdgcn_readlane(incl, 63);
    int at;
    if (BY_SEQ) {
      at = key - b0 < 64 ? key - b0 : -1;
    } else {
      const unsigned long long m = __ballot(base + incl > key);
      at = m ? __ffsll(m) - 1 : -1;
    }
    if (at >= 0) {
      w.b = b0 + at;
      w.nsplit = __builtin_amdgcn_readlane(n, at);
      w.first = base + __builtin_amdgcn_readlane(incl, at) - w.nsplit;
      return w;
    }
    base += sum;
  }
  return w;
}

// A step's stored bytes as a lane holds them.
template <int HD> struct Raw {
  unsigned k[2][HD / 32];      // the lane's dimensions of its two keys
  unsigned v[C4<HD>::VUNIT / 4];
  u32x2 ks, vs;                // scales of 8 keys each
};

// A column's reference is raised, and its accumulators rescaled, when a score
// exceeds it by more than this (log2): probabilities are then at most 2^RESCALE, whose fp16
// rounding is relative like that of those below one.  At 0 some one of a block's 16 columns has a
// new maximum in half of the steps of a 1300-key sequence, and the rescale is a
// third of a step's instructions.
constexpr float RESCALE = 8.0f;

constexpr int NWAVE = 4;

// KW waves of the workgroup share columns and take turns along the keys; the
// others have the columns after theirs.
template <class T, int HD, int CB, int KW>
__global__ __launch_bounds__(64 * NWAVE, CB == 1 && sizeof(T) == 2 ? 4 : CB == 4 ? 1 : 2) void attn4_columns_kernel(Attn4Args a) {
  using L = C4<HD>;
  constexpr int KF = HD / 32;                 // score fragments of a key
  constexpr int VF = HD / 16;                 // value fragments of a unit
  constexpr int CW = NWAVE / KW;              // waves along the columns
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), lg = lane >> 4, lc = lane & 15;
  const int kw = w % KW;
  const int h = blockIdx.x % a.hkv, cg = blockIdx.x / a.hkv, slot = blockIdx.y;
  const Work wk = find_work<false>(a, slot);
  if (wk.b < 0) return;
  const int b = __builtin_amdgcn_readfirstlane(wk.b);
  const int grp = a.hq / a.hkv, c0 = (cg * CW + w / KW) * 16 * CB;
  const int t0 = wk.nsplit == 1 ? 0 : (slot - wk.first) * wk.chunk, ts = t0 + kw;

  // What needs no length is requested before the lengths are waited for: the
  // pages of this wave's steps ts, ts + KW, ..., 64 at a time, one per lane, and the queries.
  const int* row = a.table + (size_t)b * a.width;
  auto pages_from = [&](int t) __attribute__((always_inline)) {
    return row[(int)min(((long long)(t + lane * KW) * STEP) >> a.c.psh, (long long)a.width - 1)];
  };
  int pages = pages_from(ts);
  // column c of the key head: query row c / grp of head h grp + c % grp;
  // columns past the last one repeat it and are not stored
  const long qrows = (long)a.batch * a.G;
  Frag<T> qf[CB][KF];
#pragma unroll
  for (int cb = 0; cb < CB; ++cb) {
    const int c = min(c0 + cb * 16 + lc, a.G * grp - 1);
    const T* q = (const T*)a.Q + ((size_t)(h * grp + c % grp) * qrows + (size_t)b * a.G + c / grp) * HD + lg * (HD / 4);
#pragma unroll
    for (int s = 0; s < KF; ++s) frag_load(qf[cb][s], q + 8 * s);
  }
  const SeqView v = seq_view(a, b);
  const int ncol = v.rows * grp;
  if (c0 >= ncol) return;                     // the whole workgroup where its waves meet below
  const int t1 = wk.nsplit == 1 ? v.steps : min(t0 + wk.chunk, v.steps), te = min(t1, v.steps1);
  // -1: a page that the cache does not have
  auto page_at = [&](int n) __attribute__((always_inline)) {
    const int p = __builtin_amdgcn_readlane(pages, n);
    return p < a.c.n_pages ? p : -1;
  };

  const int Tp = 1 << a.c.psh;
  const size_t pb = L::page_bytes(Tp);
  const uint8_t* pool = a.c.data + (size_t)h * pb;
  const size_t page_stride = pb * a.c.hkv;
  // the lane's place in a step: its two keys' rows, its value unit, their scales
  const int koff = key_row(0, lc) * L::KROW + lg * (HD / 8);
  const int voff = L::voff(Tp) + lg * L::VBLK + lc * L::VUNIT;
  const int ksoff = L::ksoff(Tp) + (lc >> 2) * L::SBLK + (lg * (HD / 4) / 32) * 8;
  const int vsoff = L::vsoff(Tp) + lg * L::SBLK + (lc * (HD / 16) / 32) * 8;
  Raw<HD> raw;
  auto load_keys = [&](int t, int page) __attribute__((always_inline)) {
    const int kp = (t * STEP) & (Tp - 1);
    const uint8_t* p = pool + (size_t)page * page_stride;
    const uint8_t* kr = p + kp * L::KROW + koff;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) __builtin_memcpy(raw.k[kb], __builtin_assume_aligned(kr + 4 * kb * L::KROW, HD / 8), HD / 8);
    raw.ks = *(const u32x2*)(p + (kp >> 3) * L::SBLK + ksoff);
  };
  auto load_values = [&](int t, int page) __attribute__((always_inline)) {
    const int kp = (t * STEP) & (Tp - 1);
    const uint8_t* p = pool + (size_t)page * page_stride;
    __builtin_memcpy(raw.v, __builtin_assume_aligned(p + (kp >> 3) * L::VBLK + voff, 16), L::VUNIT);
    raw.vs = *(const u32x2*)(p + (kp >> 3) * L::SBLK + vsoff);
  };

  f32x4 o[CB][VF];
  float m_run[CB], l_run[CB];
#pragma unroll
  for (int cb = 0; cb < CB; ++cb) {
    m_run[cb] = M_NONE;
    l_run[cb] = 0.f;
#pragma unroll
    for (int j = 0; j < VF; ++j) o[cb][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  // sc[cb][kb][e]: raw score of key 8 lg + 4 kb + e, column lc
  f32x4 sc[CB][2];
  Frag<T> pf[CB];
  auto clear = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) sc[cb][0] = sc[cb][1] = f32x4{0.f, 0.f, 0.f, 0.f};
  };
  // the s-th fragments of a step's two key blocks
  auto score = [&](const Frag<T> (&k)[2], int s) __attribute__((always_inline)) {
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
      sc[cb][0] = mfma8(k[0], qf[cb][s], sc[cb][0]);
      sc[cb][1] = mfma8(k[1], qf[cb][s], sc[cb][1]);
    }
  };
  auto value = [&](const Frag<T>& v, int j) __attribute__((always_inline)) {
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) o[cb][j] = mfma8(v, pf[cb], o[cb][j]);
  };
  // online softmax of the scores, the first `valid` keys of which count
  auto softmax = [&](int valid) __attribute__((always_inline)) {
    if (valid < STEP) {
      const int n = valid - 8 * local_value(lg);
#pragma unroll
      for (int cb = 0; cb < CB; ++cb)
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (4 * kb + e >= n) sc[cb][kb][e] = -INFINITY;
    }
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
      float m = -INFINITY;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int e = 0; e < 4; ++e) m = fmaxf(m, sc[cb][kb][e]);
      m *= a.scale_log2;
      // a lane looks at its own keys; only where one exceeds its column's
      // maximum do the four lanes of a column compare theirs.  The branch
      // is the wave's, the decision each column's (alpha = 1 leaves it as it is).
      if (__ballot(m > m_run[cb] + RESCALE)) {
        const float mc = max_groups(m);
        const float mn = mc > m_run[cb] + RESCALE ? mc : m_run[cb];
        const float alpha = __builtin_amdgcn_exp2f(m_run[cb] - mn);
        m_run[cb] = mn;
        l_run[cb] *= alpha;
#pragma unroll
        for (int j = 0; j < VF; ++j) o[cb][j] *= alpha;
      }
      float ls = 0.f;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float p = __builtin_amdgcn_exp2f(fmaf(sc[cb][kb][e], a.scale_log2, -m_run[cb]));
          ls += p;
          pf[cb].v[4 * kb + e] = (T)p;
        }
      l_run[cb] += ls;
    }
  };

  // One buffer is enough: the next step's keys are requested when this one's
  // are expanded, before its softmax, and its values after P V.
  int page = page_at(0);
  if (ts < te) {
    load_keys(ts, max(page, 0));
    load_values(ts, max(page, 0));
  }
  int n = 0;                                  // steps of `pages` already requested
  int keys = 0;                               // more than 0: the wave had a key (one scalar maximum a step)
  for (int t = ts; t < te; t += KW) {
    // a page that the cache does not have: none of its keys count
    const int valid = page < 0 ? 0 : v.len - t * STEP;
    keys = max(keys, valid);
    if (++n == 64) {
      pages = pages_from(t + KW);
      asm volatile("" : "+v"(pages));         // waits for them here, not in every step
      n = 0;
    }
    page = page_at(n);
    clear();
    const float ks[2] = {scale_of(raw.ks[0], lc & 3), scale_of(raw.ks[1], lc & 3)};
#pragma unroll
    for (int i = 0; i < KF; ++i) {
      Frag<T> k[2];
      frag_codes(k[0], raw.k[0][i], ks[0]);
      frag_codes(k[1], raw.k[1][i], ks[1]);
      score(k, i);
    }
    load_keys(min(t + KW, te - 1), max(page, 0));     // past the last step: not used
    softmax(valid);
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
    load_values(min(t + KW, te - 1), max(page, 0));
  }

  // fresh steps, in the same rotation
  int t = ts;
  if (t < v.steps1) t += (v.steps1 - t + KW - 1) / KW * KW;
  for (; t < t1; t += KW) {
    const int k0 = (t - v.steps1) * STEP, f0 = b * a.fstride + k0, valid = v.nfresh - k0;
    keys = 1;
    // every fragment of the keys, then of the values, is requested before the
    // first is used; keys past the end read the last one's, masked below
    Frag<T> k[KF][2];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      const T* kr = (const T*)a.K2 + ((size_t)h * a.ld2 + f0 + min(key_row(kb, lc), valid - 1)) * HD + lg * (HD / 4);
#pragma unroll
      for (int i = 0; i < KF; ++i) frag_load(k[i][kb], kr + 8 * i);
    }
    clear();
#pragma unroll
    for (int i = 0; i < KF; ++i) score(k[i], i);
    Frag<T> vf[VF];
    const T* vr = (const T*)a.Vt2 + ((size_t)h * HD + lc * VF) * a.ld2 + f0 + min(8 * lg, (valid - 1) & ~7);
#pragma unroll
    for (int j = 0; j < VF; ++j) frag_load(vf[j], vr + (size_t)j * a.ld2);
    softmax(valid);
    if (valid < STEP) {
#pragma unroll
      for (int j = 0; j < VF; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (8 * lg + i >= valid) vf[j].v[i] = (T)0.f;
    }
#pragma unroll
    for (int j = 0; j < VF; ++j) value(vf[j], j);
  }

  // o[cb][j][e]: dimension (4 lg + e) VF + j of column lc.
  using OT = typename OutOf<T>::type;
  auto out_row = [&](int col) __attribute__((always_inline)) {
    return (OT*)a.O + ((size_t)b * a.G + col / grp) * ((size_t)a.hq * HD) + (size_t)(h * grp + col % grp) * HD;
  };
  auto part_row = [&](int col) __attribute__((always_inline)) { return ((size_t)slot * a.hkv + h) * ((size_t)a.G * grp) + col; };
#pragma unroll
  for (int cb = 0; cb < CB; ++cb) {
    l_run[cb] = sum_groups(l_run[cb]);
    m_run[cb] = fmaxf(m_run[cb], keys > 0 ? M_KEYS : M_NONE);
  }
  if constexpr (KW == 1) {
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
      const int col = c0 + cb * 16 + lc;
      if (col >= ncol) continue;
      OT* out = out_row(col);
      const size_t at = part_row(col);
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int j = 0; j < VF; j += 4) {
          const f32x4 x = {o[cb][j][e], o[cb][j + 1][e], o[cb][j + 2][e], o[cb][j + 3][e]};
          if (wk.nsplit == 1) store_row4<OT>(out + (4 * lg + e) * VF + j, x, final_sum(l_run[cb], m_run[cb]));
          else *(f32x4*)(a.Opart + at * HD + (4 * lg + e) * VF + j) = x;
        }
      if (wk.nsplit > 1 && lg == 0) *(float2*)(a.ML + at * 2) = make_float2(m_run[cb], l_run[cb]);
    }
  } else {
    // Join the waves: the columns' maxima, then sums and accumulators relative
    // to them, half of the dimensions at a time.
    constexpr int HH = HD / 2;
    __shared__ float sm[KW][16 * CB], sl[KW][16 * CB], smax[16 * CB];
    __shared__ __attribute__((aligned(16))) float so[KW][16][HH + 4];
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
      if (lg == 0) sm[w][cb * 16 + lc] = m_run[cb];
    __syncthreads();
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
      const int cols = min(ncol - c0 - cb * 16, 16);
      if (cols <= 0) break;
      float M = M_NONE;
#pragma unroll
      for (int i = 0; i < KW; ++i) M = fmaxf(M, sm[i][cb * 16 + lc]);
      const float f = __builtin_amdgcn_exp2f(m_run[cb] - M);
      if (lg == 0) {
        sl[w][cb * 16 + lc] = l_run[cb] * f;
        if (w == 0) smax[cb * 16 + lc] = M;
      }
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        if (cb + half) __syncthreads();
        if (lg >> 1 == half && lc < cols) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int j = 0; j < VF; j += 4)
              *(f32x4*)&so[w][lc][(4 * (lg & 1) + e) * VF + j] =
                  f32x4{o[cb][j][e] * f, o[cb][j + 1][e] * f, o[cb][j + 2][e] * f, o[cb][j + 3][e] * f};
        }
        __syncthreads();
        for (int i = tid; i < cols * (HH / 4); i += 64 * NWAVE) {
          const int c = i / (HH / 4), d = i % (HH / 4) * 4, col = c0 + cb * 16 + c;
          float l = 0.f;
          f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int k = 0; k < KW; ++k) {
            l += sl[k][cb * 16 + c];
            x += *(const f32x4*)&so[k][c][d];
          }
          if (wk.nsplit == 1) {
            store_row4<OT>(out_row(col) + half * HH + d, x, final_sum(l, smax[cb * 16 + c]));
          } else {
            const size_t at = part_row(col);
            *(f32x4*)(a.Opart + at * HD + half * HH + d) = x;
            if (half == 0 && d == 0) *(float2*)(a.ML + at * 2) = make_float2(smax[cb * 16 + c], l);
          }
        }
      }
    }
  }
}

// ---------------------------------------------------------------------------
// Row kernel: many columns (fp16, 128 dimensions).  Eight waves of 32 columns, two to
// a SIMD, share tiles of 64 keys, and what the column kernel spends on
// expanding a tile for every 32 columns is spent once for 256:
//   * Scores on the codes themselves.  The fp4 x fp6 MFMA (16x16x128, block scales) takes
//     a key's 32 codes of a lane and their scale byte as they are stored, at the
//     rate of an fp16 16x16x32, so four times its work.  A query is the sum of four
//     e2m3 terms per 32 dimensions, each term's scale a power of two:
//       q = t1 + t2 + t3 + t4 + r,  |r| <= 2^-17 s1,  s1 = the scale of t1, max |q| > 3.75 s1,
//     an error of at most 2^-18.9 of the largest element of the 32, less than the fp32 sums may be
//     off by.  Four MFMAs do what four fp16 ones would, and no key is expanded.  (Three terms:
//     2^-13.9, which is more than the fp16 probabilities' rounding where scores are large or one of the 32
//     elements outweighs the others; 39.2 us in place of 40.7 for 8 sequences of 512 + 256 keys, 174 in
//     place of 190 for 8 of 5376.)  The queries
//     carry the softmax's factor, and the MFMA starts from minus the column's reference,
//     so that a score comes out as the exponent of its probability.
//   * Values are expanded by all eight waves, one tile ahead, into the operand
//     order of P V in LDS, so that every fragment is one conflict-free 16-byte read.
//   * The probabilities' sum is a row of ones in P V.
//   * The two waves of a SIMD are half a tile apart, with a barrier after each half: while
//     one multiplies, the other one exponentiates and expands.
// Measured, 32/32 heads, 256 rows, back to back (the clock falls by a tenth in the longer ones): 8 sequences of
// 5376 keys 190 to 200 us (0.95 to 0.90 PF/s; a large fp16 library product reaches 1.22 on this GPU),
// 8 of 512 cached and 256 fresh keys 40 us, 16 of 1344 and 256 132 to 159.  Of the cycles the
// matrix pipes are busy in 56 %, a wave waits in 21 %.  A tile takes about 3900 in both halves: P V 730,
// scores 790, exponentials and loads 600 to 800, softmax 300, expansion 330, LDS stores 210 to
// 340, and the rest waiting at the barriers, for the halves are not equally long.
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

constexpr int RW = 8;
constexpr int NST = 3;       // stages: the tile whose scores are made, the one before it (its values), the next one

struct RowStage {
  u32x4 v[2 * 8 * 64];       // value fragments [half][j][lane]
  u32x4 k[4 * 64];           // codes [kb][lane]
  uint16_t ks[128];          // a lane's scales of the four key blocks
};
// a tile of fresh keys: fragments [kb][s][lane], [half][j][lane]
struct FreshStage {
  u32x4 v[2 * 8 * 64];
  u32x4 k[4 * 4 * 64];
};

// all LDS traffic of this wave done, then the barrier; loads in flight stay so
__device__ __forceinline__ void lds_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

__global__ __launch_bounds__(64 * RW, 2) void attn4_rows_kernel(Attn4Args a) {
  constexpr int HD = 128, CB = 2, KF = HD / 32, VF = HD / 16, NT = 64 * RW;
  using L = C4<HD>;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), lg = lane >> 4, lc = lane & 15;
  const int h = blockIdx.x % a.hkv, cg = blockIdx.x / a.hkv;
  const int b = a.sorted ? __builtin_amdgcn_readfirstlane(by_length(a, blockIdx.y)) : (int)blockIdx.y;
  const int grp = a.hq / a.hkv, c0 = (cg * RW + w) * 16 * CB;
  // The queries and the first pages are requested before the lengths are waited for.
  const long qrows = (long)a.batch * a.G;
  auto query = [&](int cb) __attribute__((always_inline)) {
    const int c = min(c0 + cb * 16 + lc, a.G * grp - 1);
    return (const f16*)a.Q + ((size_t)(h * grp + c % grp) * qrows + (size_t)b * a.G + c / grp) * HD;
  };
  // a lane's 32 dimensions from 32 lg: the fragments of the fresh keys' products, and
  // the elements of the terms for the cached ones
  Frag<f16> qf[CB][KF];
#pragma unroll
  for (int cb = 0; cb < CB; ++cb)
#pragma unroll
    for (int i = 0; i < KF; ++i) frag_load(qf[cb][i], query(cb) + lg * 32 + 8 * i);
  const int* row = a.table + (size_t)b * a.width;
  // a lane's page of half tile pbase + lane, 64 at a time
  int pbase = 0;
  auto fetch_pages = [&]() __attribute__((always_inline)) {
    return row[(int)min(((long long)(pbase + lane) * 32) >> a.c.psh, (long long)a.width - 1)];
  };
  int page0 = fetch_pages();
  const SeqView v = seq_view(a, b);
  const int ncol = v.rows * grp;
  if (cg * RW * 16 * CB >= ncol) return;
  const bool live = c0 < ncol;                // other waves fill and wait with the rest
  const int te = v.steps1, tf = v.steps - te; // cached and fresh tiles
  const int Tp = 1 << a.c.psh;
  const size_t pb = L::page_bytes(Tp);
  const uint8_t* pool = a.c.data + (size_t)h * pb;
  const size_t page_stride = pb * a.c.hkv;
  constexpr size_t STAGE = sizeof(RowStage) > sizeof(FreshStage) ? sizeof(RowStage) : sizeof(FreshStage);
  constexpr size_t OUT = 16 * (HD * 2 + 16);      // a wave's 16 output rows, on their way out
  __shared__ __attribute__((aligned(16))) char lds[NST * STAGE > RW * OUT ? NST * STAGE : RW * OUT];
  __shared__ int simd_of[RW];
  RowStage* st = (RowStage*)lds;
  FreshStage* fs = (FreshStage*)lds;

  // ---- filling
  // What a thread fetches of a tile, in loads that every thread makes of every
  // tile (a branch around one would make the compiler wait for all of them): the
  // value unit (block vblk of the half that its wave has, unit u), of which it
  // expands byte vbyte of each key; and 16 bytes of codes (waves 0-3: key block w)
  // or of key scales (waves 4, 5: half w & 1; 6, 7 the same, unused).
  struct Raw2 {
    u32x4 v[2];
    u32x2 vs;
    u32x4 k;
  };
  // (addresses of the global address space by name: chosen between two pages, the
  // compiler would not know them for such, and a flat load waits for LDS as well)
  typedef const __attribute__((address_space(1))) uint8_t* gbytes;
  typedef const __attribute__((address_space(1))) u32x4* gvec4;
  typedef const __attribute__((address_space(1))) u32x2* gvec2;
  const int vhalf = w & 1, vblk = (tid >> 4) & 3, u = tid & 15, vbyte = w >> 1;
  const int khalf = w < 4 ? w >> 1 : w & 1;
  const unsigned voff = (unsigned)(L::voff(Tp) + vblk * L::VBLK + u * L::VUNIT);
  const unsigned vsoff = (unsigned)(L::vsoff(Tp) + vblk * L::SBLK + (u >> 2) * 8);
  const unsigned koff = w < 4 ? (unsigned)(key_row(w & 1, lc) * L::KROW + lg * 16)
                              : (unsigned)(L::ksoff(Tp) + (lc >> 2) * L::SBLK + lg / 2 * 16);
  // What the tiles' addresses and valid keys need of the scalar unit is made by
  // the lanes, for 32 tiles at once: where a half's codes begin, of a page that is there
  // (position kp: kp KROW bytes of keys, as many of values, kp SBLK / 8 of scales).
  static_assert(L::VBLK == 8 * L::KROW, "keys and values advance alike");
  unsigned alo, ahi;
  int avalid;
  auto place = [&](int page) __attribute__((always_inline)) {
    const unsigned k0 = (unsigned)(pbase + lane) * 32u;      // of the last tiles' lanes, up to 2^31 and some
    const bool ok = page >= 0 && page < a.c.n_pages;
    avalid = ok ? min(max((int)((unsigned)v.len - k0), 0), 32) : 0;
    const uintptr_t p = (uintptr_t)(pool + (size_t)(ok ? page : 0) * page_stride + (size_t)((k0 & (Tp - 1)) * L::KROW));
    alo = (unsigned)p;
    ahi = (unsigned)(p >> 32);
  };
  place(page0);
  // the tile's bytes into r; valid keys of the two halves, packed
  auto load = [&](Raw2& r, int t) __attribute__((always_inline)) {
    int n = 2 * t - pbase;
    if (n >= 64) {
      pbase = 2 * t;
      place(fetch_pages());
      asm volatile("" : "+v"(alo));           // waits for them here, not in every tile
      n = 0;
    }
    auto at = [&](int i) __attribute__((always_inline)) {
      return (gbytes)((uintptr_t)(unsigned)__builtin_amdgcn_readlane((int)alo, i) |
                      (uintptr_t)(unsigned)__builtin_amdgcn_readlane((int)ahi, i) << 32);
    };
    const int kv = (t * TILE + 32 * vhalf) & (Tp - 1), kk = (t * TILE + 32 * khalf) & (Tp - 1);
    constexpr int BACK = L::KROW - L::SBLK / 8;   // scales advance by so much less
    const gbytes q = at(n + vhalf), qk = at(n + khalf);
    const unsigned vo = local_value(voff), so = local_value(vsoff) - kv * BACK, ko = local_value(koff) - (w < 4 ? 0 : kk * BACK);
    r.v[0] = *(gvec4)(q + vo);
    r.v[1] = *(gvec4)(q + 16 + vo);
    r.vs = *(gvec2)(q + so);
    r.k = *(gvec4)(qk + ko);
    return __builtin_amdgcn_readlane(avalid, n) | __builtin_amdgcn_readlane(avalid, n + 1) << 16;
  };
  auto fill = [&](RowStage& s, const Raw2& r, int val) __attribute__((always_inline)) {
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
    u32x4* d = s.v + ((vhalf * VF + 2 * vbyte) * 64 + vblk * 16 + u);
    d[0] = __builtin_bit_cast(u32x4, lo.v);
    d[64] = __builtin_bit_cast(u32x4, hi.v);
    if (w < 4) {
      s.k[w * 64 + lane] = r.k;
    } else if (w < 6) {
      // the lane's two keys of this half: bytes lc & 3 of both words of its 8
      const unsigned a0 = lg & 1 ? r.k[2] : r.k[0], a1 = lg & 1 ? r.k[3] : r.k[1];
      s.ks[2 * lane + khalf] = (uint16_t)__builtin_amdgcn_perm(a1, a0, 0x0c0c0400u + (unsigned)(lc & 3) * 0x0101u);
    }
  };

  // ---- this wave's columns
  Raw2 raw;
  int val = 0;
  // tiles past the last one are loaded as the last one, and not used
  auto load_at = [&](int t) __attribute__((always_inline)) { return load(raw, min(t, te - 1)); };
  if (te) val = load_at(0);

  f32x4 o[CB][VF], l[CB];
  // minus the column's reference, four times as the MFMA's addend; a score above
  // it by more than thr raises the reference (the first one does whatever it is)
  f32x4 ref[CB];
  float thr[CB];
#pragma unroll
  for (int cb = 0; cb < CB; ++cb) {
    l[cb] = ref[cb] = f32x4{0.f, 0.f, 0.f, 0.f};
    thr[cb] = M_NONE;
#pragma unroll
    for (int j = 0; j < VF; ++j) o[cb][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  f32x4 sc[CB][4];      // [kb][e]: key 32 (kb / 2) + 8 lg + 4 (kb & 1) + e, column lc, relative to its reference
  Frag<f16> ones;
#pragma unroll
  for (int e = 0; e < 8; ++e) ones.v[e] = (f16)1.f;
  // probabilities: masks the scores, and sees that none exceeds its column's
  // reference by too much
  Frag<f16> pf[CB][2];
  int keys = 0;         // not 0: a tile had a key
  auto softmax = [&](int val) __attribute__((always_inline)) {
    keys |= val;
    if (val != (32 | 32 << 16)) {
      const int k0 = 8 * local_value(lg), n0 = (val & 0xffff) - k0, n1 = (val >> 16) - k0;
#pragma unroll
      for (int cb = 0; cb < CB; ++cb)
#pragma unroll
        for (int kb = 0; kb < 4; ++kb)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (4 * (kb & 1) + e >= (kb < 2 ? n0 : n1)) sc[cb][kb][e] = -INFINITY;
    }
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
      float m = -INFINITY;
#pragma unroll
      for (int kb = 0; kb < 4; ++kb)
#pragma unroll
        for (int e = 0; e < 4; ++e) m = fmaxf(m, sc[cb][kb][e]);
      if (__ballot(m > thr[cb])) {
        const float mc = max_groups(m);
        const bool up = mc > thr[cb];
        const float by = up ? mc : 0.f;
        const float alpha = thr[cb] < 0.f ? 1.f : __builtin_amdgcn_exp2f(-by);   // nothing to rescale at first
        thr[cb] = up ? RESCALE : thr[cb];
        ref[cb] -= by;
        l[cb] *= alpha;
#pragma unroll
        for (int j = 0; j < VF; ++j) o[cb][j] *= alpha;
#pragma unroll
        for (int kb = 0; kb < 4; ++kb) sc[cb][kb] -= by;
      }
#pragma unroll
      for (int kb = 0; kb < 4; ++kb)
#pragma unroll
        for (int e = 0; e < 4; ++e) pf[cb][kb >> 1].v[4 * (kb & 1) + e] = (f16)__builtin_amdgcn_exp2f(sc[cb][kb][e]);
    }
  };
  // P V.  The fragments of the first half are requested together, each one of the
  // second half in the place of its predecessor: left to itself the scheduler asks
  // for a fragment right before its MFMA.
  auto values = [&](const u32x4* vs) __attribute__((always_inline)) {
    Frag<f16> f[VF];
#pragma unroll
    for (int j = 0; j < VF; ++j) f[j].v = __builtin_bit_cast(f16x8, vs[j * 64 + lane]);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
#pragma unroll
      for (int j = 0; j < VF; ++j) {
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) o[cb][j] = mfma8(f[j], pf[cb][half], o[cb][j]);
        if (half == 0) f[j].v = __builtin_bit_cast(f16x8, vs[(VF + j) * 64 + lane]);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) l[cb] = mfma8(ones, pf[cb][half], l[cb]);
    }
  };
  // Which of the two waves on its SIMD this one is: only the schedule depends on it.
  if (lane == 0) simd_of[w] = __builtin_amdgcn_s_getreg((1 << 11) | (4 << 6) | 4) & 3;   // SIMD_ID of HW_ID
  lds_barrier();
  int turn = 0;
  for (int i = 0; i < w; ++i) turn += simd_of[i] == simd_of[w];
  turn = __builtin_amdgcn_readfirstlane(turn & 1);

  // Tiles 0 .. nt - 1 of one kind.  score(s) makes the scores of the tile in stage s,
  // prep(s, i, n) expands tile i into it (n: its valid keys), requests tile i + 1
  // and returns that one's valid keys, vals(s) are the stage's value fragments.  A tile's
  // values are read right before the scores of the next one, so that its stage is free for
  // the third one after it.
  auto up = [](int s) __attribute__((always_inline)) { return s == NST - 1 ? 0 : s + 1; };
  auto pipeline = [&](int nt, int val, auto score, auto prep, auto vals) __attribute__((always_inline)) {
    int cur = val, next = prep(0, 0, val), after = 0;
    lds_barrier();
    if (!live) {
      for (int i = 1, s = 1; i <= nt; ++i, s = up(s)) {
        next = prep(s, i, next);
        lds_barrier();
        lds_barrier();
      }
      lds_barrier();
    } else {
      // the second of a SIMD's waves begins half a tile later, and so expands a tile further ahead
      if (turn) {
        after = prep(1, 1, next);
        lds_barrier();
      }
      score(0);
      for (int i = 1, s = 1, sp = 1 + turn, sv = 0;; ++i) {
        lds_barrier();
        softmax(cur);
        cur = next;
        const int n = prep(sp, i + turn, turn ? after : next);
        next = turn ? after : n;
        after = n;
        lds_barrier();
        values(vals(sv));
        if (i == nt) break;
        score(s);
        sv = s; s = up(s); sp = up(sp);
      }
      if (!turn) lds_barrier();
    }
    lds_barrier();                            // the stages are free
  };

  // ---- fresh tiles first (the first cached one is on its way): fp16 keys and
  // values, brought into operand order by all waves
  if (tf) {
    constexpr int KC = 4 * KF * 64 / NT, VC = 2 * VF * 64 / NT;   // 16-byte chunks of a thread
    u32x4 fk[KC], fv[VC];
    // valid keys of tile i; tiles past the last one are taken as the last one
    auto left = [&](int i) __attribute__((always_inline)) { return v.nfresh - min(i, tf - 1) * TILE; };
    auto packed = [&](int n) __attribute__((always_inline)) { return min(n, 32) | min(max(n - 32, 0), 32) << 16; };
    auto fload = [&](int i) __attribute__((always_inline)) {
      const int n = left(i), k0 = v.nfresh - n;
#pragma unroll
      for (int e = 0; e < KC; ++e) {
        const int c = e * NT + tid, kb = c / (64 * KF), s = c / 64 % KF;
        const int key = min(32 * (kb >> 1) + key_row(kb & 1, lc), n - 1);
        fk[e] = *(const u32x4*)((const f16*)a.K2 + ((size_t)h * a.ld2 + (size_t)b * a.fstride + k0 + key) * HD + 32 * lg + 8 * s);
      }
#pragma unroll
      for (int e = 0; e < VC; ++e) {
        const int c = e * NT + tid, half = c / (64 * VF), j = c / 64 % VF, k = 32 * half + 8 * lg;
        fv[e] = *(const u32x4*)((const f16*)a.Vt2 + ((size_t)h * HD + lc * VF + j) * a.ld2 + (size_t)b * a.fstride + k0 + min(k, (n - 1) & ~7));
      }
    };
    auto prep = [&](int stage, int i, int) __attribute__((always_inline)) {
      FreshStage& s = fs[stage];
      const int n = left(i);
#pragma unroll
      for (int e = 0; e < KC; ++e) s.k[e * NT + tid] = fk[e];
#pragma unroll
      for (int e = 0; e < VC; ++e) {
        const int half = (e * NT + tid) / (64 * VF), k = 32 * half + 8 * lg;
        if (n < TILE) {
#pragma unroll
          for (int x = 0; x < 4; ++x) fv[e][x] &= (k + 2 * x < n ? 0xffffu : 0u) | (k + 2 * x + 1 < n ? 0xffff0000u : 0u);
        }
        s.v[e * NT + tid] = fv[e];
      }
      fload(i + 1);
      return packed(left(i + 1));
    };
    auto score = [&](int stage) __attribute__((always_inline)) {
      const FreshStage& s = fs[stage];
#pragma unroll
      for (int kb = 0; kb < 4; ++kb) {
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) sc[cb][kb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int x = 0; x < KF; ++x) {
          Frag<f16> k;
          k.v = __builtin_bit_cast(f16x8, s.k[(kb * KF + x) * 64 + lane]);
#pragma unroll
          for (int cb = 0; cb < CB; ++cb) sc[cb][kb] = mfma8(k, qf[cb][x], sc[cb][kb]);
        }
#pragma unroll
        for (int cb = 0; cb < CB; ++cb)
#pragma unroll
          for (int e = 0; e < 4; ++e) sc[cb][kb][e] = fmaf(sc[cb][kb][e], a.scale_log2, ref[cb][e]);
      }
    };
    fload(0);
    pipeline(tf, packed(left(0)), score, prep, [&](int s) __attribute__((always_inline)) { return fs[s].v; });
  }

  // ---- cached tiles
  if (te) {
    QTerms q[CB];
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) q[cb] = query_terms(qf[cb], a.scale_log2);
    auto score = [&](int stage) __attribute__((always_inline)) {
      const RowStage& s = st[stage];
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
    };
    auto prep = [&](int stage, int i, int n) __attribute__((always_inline)) {
      fill(st[stage], raw, n);
      return load_at(i + 1);
    };
    pipeline(te, val, score, prep, [&](int s) __attribute__((always_inline)) { return st[s].v; });
  }

  // ---- out, 16 rows at a time through LDS, so that whole rows are stored
  if (!live) return;
  constexpr int RB = OUT / 16;
  char* buf = lds + w * OUT;
#pragma unroll
  for (int cb = 0; cb < CB; ++cb) {
    const float sum = final_sum(l[cb][0], keys ? M_KEYS : M_NONE), inv = sum == 0.f ? 0.f : 1.0f / sum;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
#pragma unroll
      for (int j = 0; j < VF; j += 4) {
        bf16x4 y;
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = (bf16)(o[cb][j + i][e] * inv);
        *(bf16x4*)(buf + lc * RB + ((4 * lg + e) * VF + j) * 2) = y;
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
    for (int i = 0; i < 16 * (HD / 8); i += 64) {
      const int r = (i + lane) / (HD / 8), c = lane % (HD / 8), col = c0 + cb * 16 + r;
      const u32x4 x = *(const u32x4*)(buf + r * RB + c * 16);
      if (col < ncol)
        *(u32x4*)((bf16*)a.O + ((size_t)b * a.G + col / grp) * ((size_t)a.hq * HD) + (size_t)(h * grp + col % grp) * HD + c * 8) = x;
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  }
}

// Join of a sequence's chunks.  SL > 1 (many chunks of few rows): a workgroup per
// (row, head), its threads 4 dimensions of every SL-th chunk each, then over the SL through
// LDS.  SL = 1 (many rows of few chunks): a thread 4 dimensions of a row and all of its
// chunks.  U partials are requested at a time.
template <class T, int HD, int SL>
__global__ __launch_bounds__(256) void attn4_merge_kernel(Attn4Args a) {
  constexpr int TPR = HD / 4, RPB = 256 / (TPR * SL), U = SL > 1 ? 4 : 8;
  using OT = typename OutOf<T>::type;
  const int b = blockIdx.y, tid = threadIdx.x, sl = tid / TPR % SL, d = tid % TPR * 4;
  const long i = (long)blockIdx.x * RPB + tid / (TPR * SL);
  const Work wk = find_work<true>(a, b);
  if (wk.nsplit == 1) return;
  const int rows = a.resp_len ? min(max(a.resp_len[b], 0), a.G) : a.G;
  // row i of the sequence's partials: key head, column
  const int grp = a.hq / a.hkv, per = a.G * grp, h = (int)(i / per), col = (int)(i % per);
  const bool live = h < a.hkv && col < rows * grp;
  if (SL == 1 ? !live : __builtin_amdgcn_readfirstlane((int)!live)) return;
  const size_t stride = (size_t)a.hq * a.G, at = (size_t)wk.first * stride + i;
  float m = M_NONE, l = 0.f;
  f32x4 x = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = sl; s0 < wk.nsplit; s0 += SL * U) {
    float2 ml[U];
    f32x4 p[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int s = min(s0 + u * SL, wk.nsplit - 1);
      ml[u] = *(const float2*)(a.ML + (at + s * stride) * 2);
      p[u] = *(const f32x4*)(a.Opart + (at + s * stride) * HD + d);
    }
    float mn = m;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (s0 + u * SL >= wk.nsplit) ml[u] = make_float2(M_NONE, 0.f), p[u] = f32x4{0.f, 0.f, 0.f, 0.f};
      mn = fmaxf(mn, ml[u].x);
    }
    const float f = __builtin_amdgcn_exp2f(m - mn);
    l *= f;
    x *= f;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float g = __builtin_amdgcn_exp2f(ml[u].x - mn);
      l += ml[u].y * g;
      x += p[u] * g;
    }
    m = mn;
  }
  if constexpr (SL > 1) {
    __shared__ float sm[SL], slm[SL];
    __shared__ f32x4 sx[SL][TPR];
    if (d == 0) { sm[sl] = m; slm[sl] = l; }
    sx[sl][d / 4] = x;
    __syncthreads();
    if (sl) return;
    float M = M_NONE;
#pragma unroll
    for (int s = 0; s < SL; ++s) M = fmaxf(M, sm[s]);
    m = M;
    l = 0.f;
    x = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < SL; ++s) {
      const float f = __builtin_amdgcn_exp2f(sm[s] - M);
      l += slm[s] * f;
      x += sx[s][d / 4] * f;
    }
  }
  store_row4<OT>((OT*)a.O + ((size_t)b * a.G + col / grp) * ((size_t)a.hq * HD) + (size_t)(h * grp + col % grp) * HD + d, x, final_sum(l, m));
}

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
void launch_kind(Attn4Args a, hipStream_t st) {
  const Kind kind = kind_of(sizeof(T) == 4, a.batch, a.G, a.hq, a.hkv, a.hd);
  const long ncol = (long)a.G * (a.hq / a.hkv), cols = kind == Kind::COL1 ? 16 : kind == Kind::COL2 ? 32 : 256;
  const dim3 grid((unsigned)(a.hkv * ((ncol + cols - 1) / cols)), (unsigned)a.slots);
  // More workgroups than CUs: the longest sequences first, or the last ones to start are waited
  // for (16 sequences of 681 to 1971 cached and 256 fresh keys, 32 heads: 155 us, not 166).  In the
  // column kernel, several to a CU and shorter, it costs more than it gives (64 of 512 + 32
  // keys, 32 rows, 32 heads: 65 us, not 54).
  a.sorted = kind == Kind::WIDE && a.batch > 1 && (long)grid.x * a.batch > 256;
  if (kind == Kind::COL1) {
    attn4_columns_kernel<T, HD, 1, NWAVE><<<grid, 64 * NWAVE, 0, st>>>(a);
  } else if constexpr (sizeof(T) == 2) {
    if (kind == Kind::COL2) attn4_columns_kernel<T, HD, 2, NWAVE><<<grid, 64 * NWAVE, 0, st>>>(a);
    else if constexpr (HD == 128) attn4_rows_kernel<<<grid, 64 * RW, 0, st>>>(a);
    else attn4_columns_kernel<T, HD, 4, 1><<<grid, 64 * NWAVE, 0, st>>>(a);
  }
  if (a.slots > a.batch) {
    constexpr int SL = 256 / (HD / 4);
    const long rows = (long)a.G * a.hq;
    if (rows < 1024) attn4_merge_kernel<T, HD, SL><<<dim3((unsigned)rows, (unsigned)a.batch), 256, 0, st>>>(a);
    else attn4_merge_kernel<T, HD, 1><<<dim3((unsigned)((rows + SL - 1) / SL), (unsigned)a.batch), 256, 0, st>>>(a);
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
Attn4Split attn4_split(int fp32, int batch, int G, int hq, int hkv, int hd, int max_cached, int fresh) {
  const Kind kind = kind_of(fp32, batch, G, hq, hkv, hd);
  if (kind == Kind::WIDE) return Attn4Split{0, 0, batch, hd == 128 ? TILE : STEP};
  const long ncol = (long)G * (hq / hkv), groups = hkv * (kind == Kind::COL1 ? (ncol + 15) / 16 : (ncol + 31) / 32);
  const long steps = ((long)max_cached + STEP - 1) / STEP + ((fresh ? G : 0) + STEP - 1) / STEP;
  Attn4Split s{0, 2 * NWAVE, batch, STEP};
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

int launch_attn4(int fp32, const Attn4Args& a, hipStream_t st) {
  if (fp32) a.hd == 128 ? launch_kind<float, 128>(a, st) : launch_kind<float, 64>(a, st);
  else a.hd == 128 ? launch_kind<f16, 128>(a, st) : launch_kind<f16, 64>(a, st);
  return 0;
}
