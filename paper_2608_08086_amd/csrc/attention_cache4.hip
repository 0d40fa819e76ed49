// Non-causal attention over the 4-bit paged prompt cache and an optional
// fresh segment (layout: cache4.h):
//   O = softmax([q K4^T, q K2^T] / sqrt(D)) [V4; V2]
// per sequence, no mask other than key validity.  Stored elements are exact in
// fp16, so for fp16 queries the only roundings are those of the fp16 kernel
// beside it: the probabilities to fp16 and the output to bf16 (scores, running
// maximum and sum and the accumulators are fp32).
//
// Column kernel: the queries that share a key head are the columns of the
// score MFMA (16 per column block: G rows of hq / hkv heads), so a key head's
// bytes are read once for up to 16 CB of them.  A wave takes 32 keys at a time,
// its workgroup's four waves take turns along the workgroup's share of
// the keys, and their partial softmaxes are joined in LDS.
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
#include <algorithm>

#include "cache4.h"

namespace {

constexpr int NWAVE = 4;
constexpr int STEP = 32;          // keys of one step

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

// The value fragments of a unit: vf[j] dimension lc D/16 + j, 8 keys.
template <class T, int HD>
__device__ __forceinline__ void value_frags(Frag<T>* vf, const unsigned* w, const float* sc) {
  if constexpr (HD == 128) {          // one dword a key
    frag_pair<0, 0>(vf[0], vf[1], w, 2, sc);
    frag_pair<1, 1>(vf[2], vf[3], w, 2, sc);
    frag_pair<2, 2>(vf[4], vf[5], w, 2, sc);
    frag_pair<3, 3>(vf[6], vf[7], w, 2, sc);
  } else {                            // two keys a dword
    frag_pair<0, 2>(vf[0], vf[1], w, 1, sc);
    frag_pair<1, 3>(vf[2], vf[3], w, 1, sc);
  }
}

// key (of 32) of row r of score block kb
__device__ __forceinline__ int key_row(int kb, int r) { return 8 * (r >> 2) + 4 * kb + (r & 3); }

template <class T> struct OutOf { using type = bf16; };
template <> struct OutOf<float> { using type = float; };

struct SeqView {
  int len, nfresh, rows, steps1, steps, chunk, nsplit;
};

// What the lengths make of a sequence; the kernel and the merge agree on it.
__device__ __forceinline__ SeqView seq_view(const Attn4Args& a, int b) {
  SeqView v;
  const int cap = (int)min((long long)a.max_cached, (long long)a.width << a.c.psh);
  v.len = min(max(a.cached_len[b], 0), cap);
  v.rows = a.resp_len ? min(max(a.resp_len[b], 0), a.G) : a.G;
  v.nfresh = a.K2 ? v.rows : 0;
  v.steps1 = (v.len + STEP - 1) / STEP;
  v.steps = v.steps1 + (v.nfresh + STEP - 1) / STEP;
  v.chunk = max((v.steps + a.nsplit - 1) / a.nsplit, a.chunk_min);
  v.nsplit = max(1, (v.steps + v.chunk - 1) / v.chunk);
  return v;
}

template <class T, int HD, int CB>
__global__ __launch_bounds__(64 * NWAVE) void attn4_columns_kernel(Attn4Args a) {
  using L = C4<HD>;
  constexpr int KF = HD / 32;                 // score fragments of a key
  constexpr int VF = HD / 16;                 // value fragments of a unit
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, lg = lane >> 4, lc = lane & 15;
  const int h = blockIdx.x % a.hkv, cg = blockIdx.x / a.hkv, b = blockIdx.y, split = blockIdx.z;
  const SeqView v = seq_view(a, b);
  const int grp = a.hq / a.hkv, ncol = v.rows * grp, c0 = cg * 16 * CB;
  const int t0 = split * v.chunk, t1 = min(t0 + v.chunk, v.steps);
  if (c0 >= ncol || (split > 0 && t0 >= v.steps)) return;

  const int Tp = 1 << a.c.psh;
  const size_t pb = L::page_bytes(Tp);
  const uint8_t* pool = a.c.data + (size_t)h * pb;
  const size_t page_stride = pb * a.c.hkv;
  const int* row = a.table + (size_t)b * a.width;
  const long qrows = (long)a.batch * a.G;

  // column c of the key head: query row c / grp of head h grp + c % grp;
  // columns past the last one repeat it and are not stored
  Frag<T> qf[CB][KF];
#pragma unroll
  for (int cb = 0; cb < CB; ++cb) {
    const int c = min(c0 + cb * 16 + lc, ncol - 1);
    const T* q = (const T*)a.Q + ((size_t)(h * grp + c % grp) * qrows + (size_t)b * a.G + c / grp) * HD + lg * (HD / 4);
#pragma unroll
    for (int s = 0; s < KF; ++s) frag_load(qf[cb][s], q + 8 * s);
  }

  f32x4 o[CB][VF];
  float m_run[CB], l_run[CB];
#pragma unroll
  for (int cb = 0; cb < CB; ++cb) {
    m_run[cb] = -INFINITY;
    l_run[cb] = 0.f;
#pragma unroll
    for (int j = 0; j < VF; ++j) o[cb][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  for (int t = t0 + w; t < t1; t += NWAVE) {
    const bool cached = t < v.steps1;
    const int k0 = (cached ? t : t - v.steps1) * STEP;
    int valid = min((cached ? v.len : v.nfresh) - k0, STEP);   // keys of this step
    Frag<T> kf[2][KF], vf[VF];
    if (cached) {
      const int page = row[k0 >> a.c.psh];
      if (page < 0 || page >= a.c.n_pages) continue;          // no such page: keys that are not there
      const uint8_t* p = pool + (size_t)page * page_stride;
      const int kp = k0 & (Tp - 1);
      // keys
      const u32x2 ks = *(const u32x2*)(p + L::ksoff(Tp) + ((kp >> 3) + (lc >> 2)) * L::SBLK + (lg * (HD / 4) / 32) * 8);
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const unsigned* kr = (const unsigned*)(p + (size_t)(kp + key_row(kb, lc)) * L::KROW + lg * (HD / 8));
        const float sc = scale_of(ks[kb], lc & 3);
#pragma unroll
        for (int s = 0; s < KF; ++s) frag_codes(kf[kb][s], kr[s], sc);
      }
      // values: keys past the end get scale 0, hence zeros, whatever is stored there
      const int blk = (kp >> 3) + lg;
      const u32x2 vs = *(const u32x2*)(p + L::vsoff(Tp) + blk * L::SBLK + (lc * (HD / 16) / 32) * 8);
      const unsigned* vu = (const unsigned*)(p + L::voff(Tp) + blk * L::VBLK + lc * L::VUNIT);
      unsigned vw[L::VUNIT / 4];
#pragma unroll
      for (int i = 0; i < L::VUNIT / 4; ++i) vw[i] = vu[i];
      float sc[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) sc[i] = 8 * lg + i < valid ? scale_of(vs[i >> 2], i & 3) : 0.f;
      value_frags<T, HD>(vf, vw, sc);
    } else {
      const int f0 = b * a.fstride + k0;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const int key = min(key_row(kb, lc), valid - 1);
        const T* kr = (const T*)a.K2 + ((size_t)h * a.ld2 + f0 + key) * HD + lg * (HD / 4);
#pragma unroll
        for (int s = 0; s < KF; ++s) frag_load(kf[kb][s], kr + 8 * s);
      }
#pragma unroll
      for (int j = 0; j < VF; ++j) {
        frag_zero(vf[j]);
        if (8 * lg < valid) {
          frag_load(vf[j], (const T*)a.Vt2 + ((size_t)h * HD + lc * VF + j) * a.ld2 + f0 + 8 * lg);
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (8 * lg + i >= valid) vf[j].v[i] = (T)0.f;
        }
      }
    }

    // sc[cb][kb][e]: key 8 lg + 4 kb + e, column lc
    f32x4 sc[CB][2];
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < KF; ++i) s = mfma8(kf[kb][i], qf[cb][i], s);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] = 8 * lg + 4 * kb + e < valid ? s[e] * a.scale_log2 : -INFINITY;
        sc[cb][kb] = s;
      }
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
      float m = -INFINITY;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int e = 0; e < 4; ++e) m = fmaxf(m, sc[cb][kb][e]);
      m = fmaxf(m_run[cb], max_groups(m));
      // a step has a valid key, so m is a number unless every score is NaN or -inf
      const float ms = m == -INFINITY ? 0.f : m;
      const float alpha = __builtin_amdgcn_exp2f(m_run[cb] - ms);
      m_run[cb] = m;
      float ls = 0.f;
      Frag<T> pf;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float p = __builtin_amdgcn_exp2f(sc[cb][kb][e] - ms);
          ls += p;
          pf.v[4 * kb + e] = (T)p;
        }
      l_run[cb] = l_run[cb] * alpha + ls;
#pragma unroll
      for (int j = 0; j < VF; ++j) {
        o[cb][j] *= alpha;
        o[cb][j] = mfma8(vf[j], pf, o[cb][j]);
      }
    }
  }

  // Join the waves: columns' (m, l) first, then the scaled accumulators.
  // o[cb][j][e]: dimension (4 lg + e) VF + j of column lc.
  __shared__ float2 sml[NWAVE][16 * CB];
  __shared__ float so[NWAVE][16][HD + 4];
#pragma unroll
  for (int cb = 0; cb < CB; ++cb) {
    l_run[cb] = sum_groups(l_run[cb]);
    if (lg == 0) sml[w][cb * 16 + lc] = make_float2(m_run[cb], l_run[cb]);
  }
  __syncthreads();
  const bool last = v.nsplit == 1;
  using OT = typename OutOf<T>::type;
#pragma unroll
  for (int cb = 0; cb < CB; ++cb) {
    float M = -INFINITY;
#pragma unroll
    for (int i = 0; i < NWAVE; ++i) M = fmaxf(M, sml[i][cb * 16 + lc].x);
    const float f = M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run[cb] - M);
    if (cb) __syncthreads();
#pragma unroll
    for (int j = 0; j < VF; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) so[w][lc][(4 * lg + e) * VF + j] = o[cb][j][e] * f;
    __syncthreads();
    for (int i = tid; i < 16 * HD; i += 64 * NWAVE) {
      const int c = i / HD, d = i % HD, col = c0 + cb * 16 + c;
      if (col >= ncol) break;
      float mm = -INFINITY, l = 0.f, x = 0.f;
#pragma unroll
      for (int k = 0; k < NWAVE; ++k) mm = fmaxf(mm, sml[k][cb * 16 + c].x);
#pragma unroll
      for (int k = 0; k < NWAVE; ++k) {
        const float2 ml = sml[k][cb * 16 + c];
        l += mm == -INFINITY ? ml.y : ml.y * __builtin_amdgcn_exp2f(ml.x - mm);
        x += so[k][c][d];
      }
      const size_t r = (size_t)b * a.G + col / grp;
      const int head = h * grp + col % grp;
      if (last) {
        ((OT*)a.O)[r * ((size_t)a.hq * HD) + (size_t)head * HD + d] = from_f32<OT>(l == 0.f ? 0.f : x / l);
      } else {
        const size_t at = ((size_t)split * qrows + r) * a.hq + head;
        a.Opart[at * HD + d] = x;
        if (d == 0) *(float2*)(a.ML + at * 2) = make_float2(mm, l);
      }
    }
  }
}

// Join of a sequence's splits: a thread owns 4 dimensions of one (row, head).
template <class T, int HD>
__global__ __launch_bounds__(256) void attn4_merge_kernel(Attn4Args a) {
  constexpr int TPR = HD / 4;
  using OT = typename OutOf<T>::type;
  const int b = blockIdx.y;
  const SeqView v = seq_view(a, b);
  if (v.nsplit == 1) return;
  const long i = (long)blockIdx.x * (256 / TPR) + threadIdx.x / TPR;
  const int d = threadIdx.x % TPR * 4;
  if (i >= (long)v.rows * a.hq) return;
  const size_t r = (size_t)b * a.G + i / a.hq;
  const int head = (int)(i % a.hq);
  const size_t stride = (size_t)a.batch * a.G * a.hq, at = r * a.hq + head;
  float M = -INFINITY;
  for (int s = 0; s < v.nsplit; ++s) M = fmaxf(M, a.ML[(s * stride + at) * 2]);
  float l = 0.f;
  f32x4 x = {0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < v.nsplit; ++s) {
    const float2 ml = *(const float2*)(a.ML + (s * stride + at) * 2);
    const float f = M == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(ml.x - M);
    l += ml.y * f;
    x += *(const f32x4*)(a.Opart + (s * stride + at) * HD + d) * f;
  }
  OT* out = (OT*)a.O + r * ((size_t)a.hq * HD) + (size_t)head * HD + d;
#pragma unroll
  for (int e = 0; e < 4; ++e) out[e] = from_f32<OT>(l == 0.f ? 0.f : x[e] / l);
}

template <class T, int HD>
void launch_columns(const Attn4Args& a, hipStream_t st) {
  const int ncol = a.G * (a.hq / a.hkv);
  auto grid = [&](int cb) { return dim3((unsigned)(a.hkv * ((ncol + 16 * cb - 1) / (16 * cb))), (unsigned)a.batch, (unsigned)a.nsplit); };
  if (ncol <= 16) attn4_columns_kernel<T, HD, 1><<<grid(1), 64 * NWAVE, 0, st>>>(a);
  else attn4_columns_kernel<T, HD, 2><<<grid(2), 64 * NWAVE, 0, st>>>(a);
  if (a.nsplit > 1) {
    const long rows = (long)a.G * a.hq, per = 256 / (HD / 4);
    attn4_merge_kernel<T, HD><<<dim3((unsigned)((rows + per - 1) / per), (unsigned)a.batch), 256, 0, st>>>(a);
  }
}

}  // namespace

int attn4_splits(int fp32, int batch, int G, int hq, int hkv, int max_cached, int fresh) {
  const long ncol = (long)G * (hq / hkv), cols = ncol <= 16 ? 16 : 32;
  const long wgs = (long)batch * hkv * ((ncol + cols - 1) / cols);
  const long steps = ((long)max_cached + STEP - 1) / STEP + ((fresh ? G : 0) + STEP - 1) / STEP;
  // two workgroups per CU, each wave at least two steps
  return (int)std::max(1L, std::min({(512 + wgs - 1) / wgs, (steps + 2 * NWAVE - 1) / (2 * NWAVE), 64L}));
}

int launch_attn4(int fp32, const Attn4Args& a, hipStream_t st) {
  if (fp32) a.hd == 128 ? launch_columns<float, 128>(a, st) : launch_columns<float, 64>(a, st);
  else a.hd == 128 ? launch_columns<f16, 128>(a, st) : launch_columns<f16, 64>(a, st);
  return 0;
}
