// Non-causal attention over a paged prompt cache and an optional fresh segment:
//   O = softmax([q K^T, q K2^T] / sqrt(D)) [V; V2]
// per sequence, no mask other than key validity, for a cache of 4 (cache4.h) or 8 (cache8.h)
// bits an element.  What depends on the cache's format F is the place of a key's and a value's
// bytes and their expansion:
//   F::dim(lg, s)          the first of the 8 dimensions of a lane's s-th query and key fragment
//   F::Lane, Raw, load_keys, load_values, keys, values   a step of the column kernel
//   F::Row                 a tile of the row kernel
// Stored elements are exact in fp16, so for fp16 queries the column kernel's only roundings are
// those of the fp16 attention of a contiguous cache: the probabilities to fp16 and the output to
// bf16 (scores, running maximum and sum and the accumulators are fp32).
//
// Column kernel: the queries that share a key head are the columns of the
// score MFMA (G rows of hq / hkv heads, 16 CB columns to a wave), and a
// wave expands what it multiplies: 32 keys at a time, straight from memory to the operands,
// the next ones requested before these are used.  The workgroup's four waves take turns
// along its share of the keys, and their partial softmaxes are joined in LDS (KW = 4); or
// each wave has columns of its own, and there is no barrier at all (KW = 1).
//
//   S^T = K Q^T   A operand: lane (lc, lg) holds key att key(lc) and D/4
//                 dimensions of it; any order of the
//                 dimensions will do as long as Q's fragments have the same.
//   O^T = V^T P^T A operand: lane (lc, lg) holds the D/16 dimensions from
//                 lc D/16 of the 8 keys 8 lg .. 8 lg + 7.
// The keys of a score block are ordered so that a lane's scores of the two
// blocks are the 8 keys that its P V operand needs.
//
// Row kernel: many columns (fp16, 128 dimensions).  Eight waves of 32 columns, two to
// a SIMD, share tiles of 64 keys, and what the column kernel spends on
// expanding a tile for every 32 columns is spent once for 256:
//   * All eight waves bring a tile's keys and values, one tile ahead, into the operand
//     order in LDS, so that every fragment is one conflict-free 16-byte read.
//   * The probabilities' sum is a row of ones in P V.
//   * The two waves of a SIMD are half a tile apart, with a barrier after each half: while
//     one multiplies, the other one exponentiates and expands.
#pragma once

#include <algorithm>
#include <climits>

#include "paged.h"

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
__device__ __forceinline__ SeqView seq_view(const PagedAttnArgs& a, int b) {
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
__device__ __forceinline__ int by_length(const PagedAttnArgs& a, int key) {
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
__device__ __forceinline__ Work find_work(const PagedAttnArgs& a, int key) {
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

// A column's reference is raised, and its accumulators rescaled, when a score
// exceeds it by more than this (log2): probabilities are then at most 2^RESCALE, whose fp16
// rounding is relative like that of those below one.  At 0 some one of a block's 16 columns has a
// new maximum in half of the steps of a 1300-key sequence, and the rescale is a
// third of a step's instructions.
constexpr float RESCALE = 8.0f;

constexpr int NWAVE = 4;

// KW waves of the workgroup share columns and take turns along the keys; the
// others have the columns after theirs.
template <class F, class T, int HD, int CB, int KW>
__global__ __launch_bounds__(64 * NWAVE, CB == 1 && sizeof(T) == 2 ? 4 : CB == 4 ? 1 : 2) void paged_columns_kernel(PagedAttnArgs a) {
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
    const T* q = (const T*)a.Q + ((size_t)(h * grp + c % grp) * qrows + (size_t)b * a.G + c / grp) * HD;
#pragma unroll
    for (int s = 0; s < KF; ++s) frag_load(qf[cb][s], q + F::dim(lg, s));
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
  const size_t pb = F::page_bytes(Tp);
  const uint8_t* pool = a.c.data + (size_t)h * pb;
  const size_t page_stride = pb * a.c.hkv;
  const typename F::Lane at(lg, lc, Tp);      // the lane's place in a step
  typename F::Raw raw;
  auto load_keys = [&](int t, int page) __attribute__((always_inline)) {
    F::load_keys(raw, at, pool + (size_t)page * page_stride, (t * STEP) & (Tp - 1));
  };
  auto load_values = [&](int t, int page) __attribute__((always_inline)) {
    F::load_values(raw, at, pool + (size_t)page * page_stride, (t * STEP) & (Tp - 1));
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
    F::template keys<T>(raw, lc, score);
    load_keys(min(t + KW, te - 1), max(page, 0));     // past the last step: not used
    softmax(valid);
    // of keys past the end zeros, whatever is stored there
    F::template values<T>(raw, valid, lg, value);
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
      const T* kr = (const T*)a.K2 + ((size_t)h * a.ld2 + f0 + min(key_row(kb, lc), valid - 1)) * HD;
#pragma unroll
      for (int i = 0; i < KF; ++i) frag_load(k[i][kb], kr + F::dim(lg, i));
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

constexpr int RW = 8;
constexpr int NST = 3;       // stages: the tile whose scores are made, the one before it (its values), the next one

// a tile of fresh keys: fragments [kb][s][lane], [half][j][lane]
struct FreshStage {
  u32x4 v[2 * 8 * 64];
  u32x4 k[4 * 4 * 64];
};

// scores of a tile in fp16: the exponents of the probabilities
template <int CB>
__device__ __forceinline__ void score_halves(f32x4 (&sc)[CB][4], const f32x4 (&ref)[CB], const FreshStage& s, int lane,
                                             const Frag<f16> (&qf)[CB][4], float scale_log2) {
  constexpr int KF = 4;
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
      for (int e = 0; e < 4; ++e) sc[cb][kb][e] = fmaf(sc[cb][kb][e], scale_log2, ref[cb][e]);
  }
}

// (addresses of the global address space by name: chosen between two pages, the
// compiler would not know them for such, and a flat load waits for LDS as well)
typedef const __attribute__((address_space(1))) uint8_t* gbytes;
typedef const __attribute__((address_space(1))) u32x4* gvec4;
typedef const __attribute__((address_space(1))) u32x2* gvec2;

// all LDS traffic of this wave done, then the barrier; loads in flight stay so
__device__ __forceinline__ void lds_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

template <class F>
__global__ __launch_bounds__(64 * RW, 2) void paged_rows_kernel(PagedAttnArgs a) {
  constexpr int HD = 128, CB = 2, KF = HD / 32, VF = HD / 16, NT = 64 * RW;
  using Row = typename F::Row;
  using Stage = typename Row::Stage;
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
  // a lane's 32 dimensions: the fragments of the fresh keys' products, and what the
  // cached ones' are made from
  Frag<f16> qf[CB][KF];
#pragma unroll
  for (int cb = 0; cb < CB; ++cb)
#pragma unroll
    for (int i = 0; i < KF; ++i) frag_load(qf[cb][i], query(cb) + F::dim(lg, i));
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
  const size_t pb = F::page_bytes(Tp);
  const uint8_t* pool = a.c.data + (size_t)h * pb;
  const size_t page_stride = pb * a.c.hkv;
  constexpr size_t STAGE = sizeof(Stage) > sizeof(FreshStage) ? sizeof(Stage) : sizeof(FreshStage);
  constexpr size_t OUT = 16 * (HD * 2 + 16);      // a wave's 16 output rows, on their way out
  __shared__ __attribute__((aligned(16))) char lds[NST * STAGE > RW * OUT ? NST * STAGE : RW * OUT];
  __shared__ int simd_of[RW];
  Stage* st = (Stage*)lds;
  FreshStage* fs = (FreshStage*)lds;

  // ---- filling
  // What a thread fetches of a tile are loads that every thread makes of every
  // tile: a branch around one would make the compiler wait for all of them.
  typename Row::Raw raw;
  const Row fetch(w, lane, Tp);
  // What the tiles' addresses and valid keys need of the scalar unit is made by
  // the lanes, for 32 tiles at once: where a half's codes begin, of a page that is there
  // (position kp: kp KROW bytes of keys, as many of values).
  unsigned alo, ahi;
  int avalid;
  auto place = [&](int page) __attribute__((always_inline)) {
    const unsigned k0 = (unsigned)(pbase + lane) * 32u;      // of the last tiles' lanes, up to 2^31 and some
    const bool ok = page >= 0 && page < a.c.n_pages;
    avalid = ok ? min(max((int)((unsigned)v.len - k0), 0), 32) : 0;
    const uintptr_t p = (uintptr_t)(pool + (size_t)(ok ? page : 0) * page_stride + (size_t)((k0 & (Tp - 1)) * Row::KROW));
    alo = (unsigned)p;
    ahi = (unsigned)(p >> 32);
  };
  place(page0);
  // the tile's bytes into r; valid keys of the two halves, packed
  auto load = [&](int t) __attribute__((always_inline)) {
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
    const int kv = (t * TILE + 32 * fetch.vhalf) & (Tp - 1), kk = (t * TILE + 32 * fetch.khalf) & (Tp - 1);
    fetch.load(raw, at(n + fetch.vhalf), at(n + fetch.khalf), kv, kk);
    return __builtin_amdgcn_readlane(avalid, n) | __builtin_amdgcn_readlane(avalid, n + 1) << 16;
  };

  // ---- this wave's columns
  int val = 0;
  // tiles past the last one are loaded as the last one, and not used
  auto load_at = [&](int t) __attribute__((always_inline)) { return load(min(t, te - 1)); };
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
        fk[e] = *(const u32x4*)((const f16*)a.K2 + ((size_t)h * a.ld2 + (size_t)b * a.fstride + k0 + key) * HD + F::dim(lg, s));
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
    auto score = [&](int stage) __attribute__((always_inline)) { score_halves<CB>(sc, ref, fs[stage], lane, qf, a.scale_log2); };
    fload(0);
    pipeline(tf, packed(left(0)), score, prep, [&](int s) __attribute__((always_inline)) { return fs[s].v; });
  }

  // ---- cached tiles
  if (te) {
    typename Row::Query q[CB];
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) q[cb] = Row::query(qf[cb], a.scale_log2);
    auto score = [&](int stage) __attribute__((always_inline)) { Row::template score<CB>(sc, ref, st[stage], lane, q, qf, a.scale_log2); };
    auto prep = [&](int stage, int i, int n) __attribute__((always_inline)) {
      fetch.fill(st[stage], raw, n);
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
__global__ __launch_bounds__(256) void paged_merge_kernel(PagedAttnArgs a) {
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

}  // namespace
